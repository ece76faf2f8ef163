// Log probabilities of given tokens with the row's entropy and its greatest alternatives, and the
// gradient of all of them with respect to the logits.
//
// logprobs_kernel streams the logits once: a warp takes one of the equal pieces of the flat run of
// 16-byte units (vocab.cuh), keeps (m, s, t) per lane and, where alternatives are asked for, the
// list of the 32 R greatest logits it has met.  A row that lies within a piece is finished by its warp; of a
// row cut between warps each writes its part, and logprobs_join_kernel joins the parts in order.
//
// The list.  A candidate is a 64-bit key: the logit's bits in the order of the numbers above the token's
// index, inverted; so keys are unique, a greater key is a greater logit or the same one at a lower
// index, and whatever order candidates come in, the result is one.  A warp compares the maximum of each
// batch with a bound below which nothing can enter; only units above it are looked at, and what
// passes goes to a buffer in shared memory, which is sorted and merged into the list when
// it holds 32 R candidates.  The bound starts as a logit that at least top_k of the first batch's
// partial maxima reach, and after each merge is the next number above the list's entry top_k (later
// tokens have higher indices: equals lose).  Of n logits about top_k ln(n / top_k) pass.
#include "vocab.cuh"

namespace estp {
namespace {

constexpr int kWarps = kVocabThreads / 32;

// ------------------------------------------------------------------ keys and lists
__device__ __forceinline__ uint32_t ordered(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);  // -0 as +0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t key_of(float z, uint32_t v) { return (uint64_t)ordered(z) << 32 | (0xFFFFFFFFu - v); }
__device__ __forceinline__ float key_logit(uint64_t k) { return unordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_token(uint64_t k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// 32 R keys a warp, key i in register i / 32 of lane i % 32 (0: none).
// One step of a bitonic network: keys i and i ^ j, the greater one to the lower index where
// bit `size` of i is clear.
template <int R>
__device__ __forceinline__ void exchange(uint64_t (&x)[R], int size, int j, int lane) {
    if (j < 32) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint64_t y = __shfl_xor_sync(0xffffffffu, x[r], j);
            const int i = r * 32 + lane;
            const bool up = ((i & size) == 0) == ((i & j) == 0);
            x[r] = (x[r] > y) == up ? x[r] : y;
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int o = r ^ (j / 32);
            if (o > r) {
                const bool down = (r * 32 & size) != 0;
                const uint64_t a = x[r], b = x[o];
                if ((a < b) != down) {
                    x[r] = b;
                    x[o] = a;
                }
            }
        }
    }
}

template <int R>
__device__ __forceinline__ void sort_keys(uint64_t (&x)[R], int lane) {
#pragma unroll
    for (int size = 2; size <= 32 * R; size *= 2)
#pragma unroll
        for (int j = size / 2; j > 0; j /= 2) exchange<R>(x, size, j, lane);
}

// The greatest 32 R of two descending lists, descending.
template <int R>
__device__ __forceinline__ void merge_keys(uint64_t (&x)[R], const uint64_t (&y)[R], int lane) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint64_t o = __shfl_sync(0xffffffffu, y[R - 1 - r], 31 - lane);
        x[r] = x[r] > o ? x[r] : o;
    }
#pragma unroll
    for (int j = 16 * R; j > 0; j /= 2) exchange<R>(x, 64 * R, j, lane);
}

// The same of two lists in shared memory, into the first.
template <int R>
__device__ __forceinline__ void merge_lists(uint64_t* to, const uint64_t* from, int lane) {
    uint64_t x[R], y[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        x[r] = to[r * 32 + lane];
        y[r] = from[r * 32 + lane];
    }
    merge_keys<R>(x, y, lane);
#pragma unroll
    for (int r = 0; r < R; ++r) to[r * 32 + lane] = x[r];
    __syncwarp();
}

// A warp's list, the candidates that wait for it, and the units that wait to be looked at (shared memory).
template <int R>
struct Candidates {
    static constexpr int kBatch = 32 * R;
    uint64_t list[kBatch];
    uint64_t waiting[kBatch + 256];  // a unit of each lane goes in before the count is looked at again
    uint32_t units[64];              // a batch adds up to 32, and 32 are taken at once
    int count, n_units;
};

// Merges waiting candidates into the list, whole batches or (all) every one.
template <int R>
__device__ __noinline__ void take_waiting(Candidates<R>* q, int top_k, bool all) {
    const int lane = threadIdx.x & 31;
    int n = q->count;
    uint64_t x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = q->list[r * 32 + lane];
    while (n >= 32 * R || (all && n > 0)) {
        const int take = n < 32 * R ? n : 32 * R;
        n -= take;
        uint64_t y[R];
#pragma unroll
        for (int r = 0; r < R; ++r) y[r] = r * 32 + lane < take ? q->waiting[n + r * 32 + lane] : 0;
        sort_keys<R>(y, lane);
        merge_keys<R>(x, y, lane);
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < R; ++r) q->list[r * 32 + lane] = x[r];
    if (lane == 0) q->count = n;
    __syncwarp();
}

// Looks at the units that wait, one a lane at a time (their second read comes from L2), and returns the
// bound for the tokens that follow all of them.
template <bool kBf16, int R>
__device__ __noinline__ float take_units(Candidates<R>* q, const char* row, int c0, int limit, int top_k, float bound,
                                         int* status) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31, n = q->n_units;
    // these units are not in the order of the tokens: an equal of the list's last may come before it or after
    uint64_t last = q->list[top_k - 1];
    float cut = last ? fmaxf(bound, key_logit(last)) : bound;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const uint32_t mine = i0 + lane < n ? q->units[i0 + lane] : 0;
        uint32_t hits = mine & ((1u << kVocabUnroll) - 1);
        const int place = c0 + (int)(mine >> kVocabUnroll);
        while (__any_sync(0xffffffffu, hits != 0)) {
            if (hits) {
                const int c = place + 32 * (__ffs(hits) - 1), first = c * per;
                hits &= hits - 1;
                if (first < limit) {  // (a lane past the segment marks its -inf where there is no bound yet)
                    const uint4 u = ld_stream(row + (int64_t)c * 16);
                    uint32_t in = 0;
#pragma unroll
                    for (int e = 0; e < per; ++e) in |= element<kBf16>(u, e) >= cut ? 1u << e : 0u;
                    if (limit - first < per) in &= (1u << (limit - first)) - 1;
                    if (last && key_logit(last) == cut) {
                        const int before = key_token(last) - first;  // tokens of the unit that come before the last
                        uint32_t equal = 0;
#pragma unroll
                        for (int e = 0; e < per; ++e) equal |= element<kBf16>(u, e) == cut ? 1u << e : 0u;
                        if (before < per) in &= ~equal | (before > 0 ? (1u << before) - 1 : 0u);
                    }
                    if (in) {
                        int at = atomicAdd(&q->count, __popc(in));
                        do {
                            const int e = __ffs(in) - 1;
                            in &= in - 1;
                            if (in_bounds(at < 32 * R + 256, status)) q->waiting[at] = key_of(element_of<kBf16>(u, e), first + e);
                            ++at;
                        } while (in);
                    }
                }
            }
            __syncwarp();
            if (q->count >= 32 * R) {
                take_waiting<R>(q, top_k, false);
                last = q->list[top_k - 1];
                if (last) cut = fmaxf(cut, key_logit(last));
            }
            __syncwarp();
        }
    }
    if (lane == 0) q->n_units = 0;
    __syncwarp();
    return last ? fmaxf(bound, unordered((uint32_t)(last >> 32) + 1)) : bound;  // the next number above it
}

// A logit that at least top_k of the warp's 32 G values reach (or -inf): the order bits from the top
// down, as far as 16 of them go.
template <int G>
__device__ __forceinline__ float reached_by(const float (&x)[G], int top_k) {
    uint32_t o[G];
#pragma unroll
    for (int g = 0; g < G; ++g) o[g] = ordered(x[g]);
    uint32_t t = 0;
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t cand = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int g = 0; g < G; ++g) n += __popc(__ballot_sync(0xffffffffu, o[g] >= cand));
        if (n >= top_k) {
            t = cand;
            if (n == top_k) break;
        }
    }
    return t <= 0x007FFFFFu ? -INFINITY : unordered(t);  // at or below the order of -inf
}

// ------------------------------------------------------------------ forward
struct LpArgs {
    VocabRows rows;
    const int32_t* targets;
    float T, c;  // c = log2(e) / T
    int top_k;
    float* logprob;
    float* entropy;
    float2* norm;
    int32_t* top_ids;
    float* top_logprobs;
    float4* part;      // [pieces][2]: m, s, t of a piece's first and last row
    uint64_t* lists;   // [pieces][2][32 R]
    int* status;
};

// A lane's share of units [c0, c1) of one row.
template <bool kBf16, int R>
__device__ __forceinline__ RowStat stream_row(const LpArgs& a, const char* row, int c0, int c1, Candidates<R>* q) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31, V = a.rows.V;
    const int limit = min(V, c1 * per);                  // tokens of the segment end here
    const int whole = min(c1, V / per);                  // units before a partial one
    LaneStat<true> st;
    float bound = -INFINITY;
    for (int b = c0; b < c1; b += 32 * kVocabUnroll) {
        uint4 v[kVocabUnroll];
        const int c = b + lane;
        if (b + 32 * kVocabUnroll <= whole) {
            const char* p = row + (int64_t)c * 16;
#pragma unroll
            for (int k = 0; k < kVocabUnroll; ++k) v[k] = ld_stream(p + k * 512);
        } else {
#pragma unroll
            for (int k = 0; k < kVocabUnroll; ++k) v[k] = load_unit<kBf16>(row, c + 32 * k, c1, V);
        }
        const float bm = units_max<kBf16, kVocabUnroll>(v);
        if constexpr (R > 0) {
            if (b == c0) {
                constexpr int G = 2 * R, w = kVocabUnroll / G;
                float g[G];
#pragma unroll
                for (int i = 0; i < G; ++i) g[i] = units_max<kBf16, w>(v + i * w);
                bound = reached_by<G>(g, a.top_k);
            }
            // a lane with candidates leaves its place and a bit for each unit that holds one
            if (__any_sync(0xffffffffu, bm >= bound)) {
                uint32_t hits = 0;
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) hits |= units_max<kBf16, 1>(v + k) >= bound ? 1u << k : 0u;
                if (hits) q->units[atomicAdd(&q->n_units, 1)] = (uint32_t)(c - c0) << kVocabUnroll | hits;
                __syncwarp();
                if (q->n_units >= 32) bound = take_units<kBf16, R>(q, row, c0, limit, a.top_k, bound, a.status);
                __syncwarp();
            }
        }
        st.template add_units<kBf16>(v, bm, a.c);
    }
    if constexpr (R > 0) {
        take_units<kBf16, R>(q, row, c0, limit, a.top_k, bound, a.status);
        take_waiting<R>(q, a.top_k, true);
    }
    return st.row(a.c);
}

// What a row's statistics and list say, written by a warp.
template <bool kBf16, int R>
__device__ __forceinline__ void write_row(const LpArgs& a, int64_t r, const char* row, const RowStat& st,
                                          const uint64_t* list) {
    const int lane = threadIdx.x & 31;
    if (!in_bounds(r >= 0 && r < a.rows.n_rows, a.status)) return;
    const bool empty = st.s == 0.f;  // (NaN is not)
    const float ls = empty ? 0.f : logf(st.s), m = pivot(st.m);
    if (lane == 0) {
        if (a.entropy) a.entropy[r] = empty ? 0.f : ls - kLn2 * (st.t / st.s);
        if (a.norm) a.norm[r] = make_float2(st.m, st.s);
        if (a.logprob) {
            const int t = a.targets[r];
            float lp = 0.f;
            if (t >= a.rows.V) {
                report(a.status, ESTP_ERR_INVALID_ARG);
                lp = NAN;
            } else if (t >= 0) {
                lp = (logit_at<kBf16>(row, t) - m) / a.T - ls;
            }
            a.logprob[r] = lp;
        }
    }
    if constexpr (R > 0) {
        const bool none = isnan(st.s);
#pragma unroll
        for (int i = lane; i < 32 * R; i += 32)
            if (i < a.top_k) {
                const uint64_t k = list[i];
                a.top_ids[r * a.top_k + i] = none ? -1 : key_token(k);
                if (a.top_logprobs) a.top_logprobs[r * a.top_k + i] = none ? NAN : (key_logit(k) - m) / a.T - ls;
            }
    }
}

// The row that all of block b's pieces lie in, or -1: its warps then join their parts themselves.
__device__ __forceinline__ int64_t row_of_block(const VocabRows& a, int64_t b) {
    const int64_t lo = b * kWarps, hi = lo + kWarps < a.pieces ? lo + kWarps : a.pieces;
    const int64_t r = piece_start(a, lo) / a.nvec;
    return (piece_start(a, hi) - 1) / a.nvec == r ? r : -1;
}

template <bool kBf16, int R>
__global__ void __launch_bounds__(kVocabThreads, kVocabBlocks) logprobs_kernel(const LpArgs a) {
    constexpr int kLists = R ? R : 1;
    __shared__ Candidates<kLists> cand[R ? kWarps : 1];
    __shared__ RowStat stats[kWarps];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the join may be scheduled
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
    const bool one_row = row_of_block(a.rows, blockIdx.x) >= 0;
    Candidates<kLists>* q = R ? &cand[warp] : nullptr;
    const int64_t start = w < a.rows.pieces ? piece_start(a.rows, w) : 0, end = w < a.rows.pieces ? piece_start(a.rows, w + 1) : 0;
    RowStat st = no_stat();
    if (R > 0 && start == end) {
        for (int i = lane; i < 32 * R; i += 32) q->list[i] = 0;
        __syncwarp();
    }
    for (int64_t u = start; u < end;) {
        const int64_t r = u / a.rows.nvec, u0 = r * a.rows.nvec;
        const int c0 = (int)(u - u0), c1 = (int)(min(end, u0 + a.rows.nvec) - u0);
        const char* row = a.rows.base + r * a.rows.ld_bytes;
        if constexpr (R > 0) {
            __syncwarp();
            for (int i = lane; i < 32 * R; i += 32) q->list[i] = 0;
            if (lane == 0) q->count = q->n_units = 0;
            __syncwarp();
        }
        if constexpr (R > 0) st = stream_row<kBf16, R>(a, row, c0, c1, q);
        else st = stream_row<kBf16, 0>(a, row, c0, c1, nullptr);
        join_lanes(st, a.c);
        if (one_row) break;
        if (c0 == 0 && c1 == a.rows.nvec) {
            write_row<kBf16, R>(a, r, row, st, R ? q->list : nullptr);
        } else {
            const int64_t slot = w * 2 + (u == start ? 0 : 1);
            if (lane == 0) a.part[slot] = make_float4(st.m, st.s, st.t, 0.f);
            if constexpr (R > 0)
                for (int i = lane; i < 32 * R; i += 32) a.lists[slot * (32 * R) + i] = q->list[i];
        }
        u = u0 + c1;
    }
    if (!one_row) return;
    // pairs of warps, the lower half taking from the upper one
    for (int half = kWarps / 2; half > 0; half /= 2) {
        if (lane == 0) stats[warp] = st;
        __syncthreads();
        if (warp < half) {
            join(st, stats[warp + half], a.c);
            if constexpr (R > 0) merge_lists<R>(q->list, cand[warp + half].list, lane);
        }
        __syncthreads();
    }
    if (warp != 0) return;
    const int64_t r = start / a.rows.nvec, lo = blockIdx.x * (int64_t)kWarps;
    const int64_t next = piece_start(a.rows, lo + kWarps < a.rows.pieces ? lo + kWarps : a.rows.pieces);
    if (start == r * a.rows.nvec && next == start + a.rows.nvec) {
        write_row<kBf16, R>(a, r, a.rows.base + r * a.rows.ld_bytes, st, R ? q->list : nullptr);
    } else {  // in the place of the block's first piece
        if (lane == 0) a.part[w * 2] = make_float4(st.m, st.s, st.t, 0.f);
        if constexpr (R > 0)
            for (int i = lane; i < 32 * R; i += 32) a.lists[w * 2 * (32 * R) + i] = q->list[i];
    }
}

// Rows cut between pieces, `warps` warps a row (1 or all of the block's): each joins the parts of every
// warps-th block of the forward in order, then pairs of warps join what they have.
template <bool kBf16, int R>
__global__ void __launch_bounds__(kVocabThreads) logprobs_join_kernel(const LpArgs a, int warps) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the parts are complete
    constexpr int kList = R ? 32 * R : 1;
    __shared__ uint64_t lists[kWarps][kList];
    __shared__ RowStat stats[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % warps;
    const int64_t r = ((int64_t)blockIdx.x * kWarps + warp) / warps;
    int64_t lo = 0, hi = 0;
    bool cut = false;
    if (r < a.rows.n_rows) {
        lo = piece_of(a.rows, r * a.rows.nvec);
        hi = piece_of(a.rows, (r + 1) * a.rows.nvec - 1);
        // one piece that held the whole row has written it, or one block
        cut = lo < hi;
        if (cut && lo / kWarps == hi / kWarps && row_of_block(a.rows, lo / kWarps) == r &&
            piece_start(a.rows, lo / kWarps * kWarps) == r * a.rows.nvec &&
            piece_start(a.rows, min((lo / kWarps + 1) * kWarps, a.rows.pieces)) == (r + 1) * a.rows.nvec)
            cut = false;
    }
    RowStat st = no_stat();
    uint64_t x[R ? R : 1];
#pragma unroll
    for (int i = 0; i < (R ? R : 1); ++i) x[i] = 0;
    auto take = [&](int64_t slot) {
        const float4 p = a.part[slot];
        if constexpr (R > 0) {
            uint64_t y[R];
#pragma unroll
            for (int i = 0; i < R; ++i) y[i] = a.lists[slot * kList + i * 32 + lane];
            merge_keys<R>(x, y, lane);
        }
        join(st, RowStat{p.x, p.y, p.z}, a.c);
    };
    if (cut) {
        for (int64_t b = lo / kWarps + sub; b <= hi / kWarps; b += warps) {
            if (row_of_block(a.rows, b) == r) {
                take(b * kWarps * 2);
            } else {
                const int64_t last = min(hi, (b + 1) * kWarps - 1);
                for (int64_t w = b * kWarps > lo ? b * kWarps : lo; w <= last; ++w)
                    take(w * 2 + (piece_start(a.rows, w) / a.rows.nvec == r ? 0 : 1));
            }
        }
    }
    if (R > 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) lists[warp][i * 32 + lane] = x[i];
        __syncwarp();
    }
    for (int half = warps / 2; half > 0; half /= 2) {  // (warps is the same for the whole grid)
        if (lane == 0) stats[warp] = st;
        __syncthreads();
        if (warp < half && cut) {
            join(st, stats[warp + half], a.c);
            if constexpr (R > 0) merge_lists<R>(lists[warp], lists[warp + half], lane);
        }
        __syncthreads();
    }
    if (cut && sub == 0) write_row<kBf16, R>(a, r, a.rows.base + r * a.rows.ld_bytes, st, lists[warp]);
}

template <bool kBf16, int R>
cudaError_t launch_forward(const LpArgs& a, cudaStream_t st) {
    logprobs_kernel<kBf16, R><<<(unsigned)((a.rows.pieces + kWarps - 1) / kWarps), kVocabThreads, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int warps = a.rows.pieces > 4 * a.rows.n_rows ? kWarps : 1;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.rows.n_rows * warps + kWarps - 1) / kWarps));
    cfg.blockDim = dim3(kVocabThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, logprobs_join_kernel<kBf16, R>, a, warps);
}

template <bool kBf16>
cudaError_t launch_forward(const LpArgs& a, cudaStream_t st) {
    if (a.top_k == 0) return launch_forward<kBf16, 0>(a, st);
    if (a.top_k <= 32) return launch_forward<kBf16, 1>(a, st);
    if (a.top_k <= 64) return launch_forward<kBf16, 2>(a, st);
    return launch_forward<kBf16, 4>(a, st);
}

// ------------------------------------------------------------------ gradient
struct LpGradArgs {
    VocabRows rows;
    char* out;
    int64_t out_bytes;  // row stride of the gradient
    const float2* norm;
    const float* entropy;
    const int32_t* targets;
    const int32_t* top_ids;
    const float* g_logprob;
    const float* g_entropy;
    const float* g_lse;
    const float* g_top;
    float T, c;
    int top_k;
    int* status;
};

constexpr int kGradUnroll = 4, kGradBlocks = 4;

// The tokens of a row that have a term of their own.
struct Named {
    int32_t id[kMaxAlternatives + 1];
    float g[kMaxAlternatives + 1];
    uint32_t bits[32];  // units of the present 1024 that hold one
};

// What the elements of a row's gradient have in common: dz_v = 2^d (A + B d), d = z c - M in the near
// frame of the maximum (vocab.cuh), or (z - m) c where it has none.
struct RowGrad {
    float m, M, A, B;
    bool framed;
};

template <bool kBf16, bool kEntropy, bool kFramed>
__device__ __forceinline__ void grad_unit(const uint4& v, const RowGrad& g, float c, float (&x)[8]) {
    const float2 c2 = make_float2(c, c), A2 = make_float2(g.A, g.A), B2 = make_float2(g.B, g.B);
    const float2 off = kFramed ? make_float2(-g.M, -g.M) : make_float2(-g.m, -g.m);
#pragma unroll
    for (int i = 0; i < (kBf16 ? 4 : 2); ++i) {
        float2 d = kFramed ? __ffma2_rn(pair<kBf16>(v, i), c2, off) : __fmul2_rn(__fadd2_rn(pair<kBf16>(v, i), off), c2);
        float2 f = A2;
        if (kEntropy) {
            d.x = max_nan(d.x, kCut);  // (2^d d is 0 for a masked token)
            d.y = max_nan(d.y, kCut);
            f = __ffma2_rn(B2, d, A2);
        }
        const float2 y = __fmul2_rn(make_float2(ex2(d.x), ex2(d.y)), f);
        x[2 * i] = y.x;
        x[2 * i + 1] = y.y;
    }
}

// Adds the terms of the named tokens of the units that `lanes` marks, of a warp's 32 from `unit` on.
template <bool kBf16>
__device__ __noinline__ void add_named(const Named& q, int n, uint32_t lanes, int unit, float* x) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31;
    while (lanes) {
        const int l = __ffs(lanes) - 1;
        lanes &= lanes - 1;
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            const int id = i < n ? q.id[i] : -1;
            uint32_t hit = __ballot_sync(0xffffffffu, id >= 0 && id / per == unit + l);
            while (hit) {
                const int j = i0 + __ffs(hit) - 1;
                hit &= hit - 1;
                if (lane == l) x[q.id[j] - (unit + l) * per] += q.g[j];
            }
        }
    }
}

// Units [chunk, stop) of a row, at most 1024; `steps` marks the 32s that hold a named token, lane l's `word` the
// units of step l.
template <bool kBf16, bool kEntropy, bool kFramed>
__device__ __forceinline__ void grad_chunk(const char* row, char* out, int chunk, int stop, int V, const RowGrad& g, float c,
                                           const Named& q, int n_named, uint32_t word, uint32_t steps) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31, whole = min(stop, V / per);  // units before a partial one
    int b = chunk;
    for (; b + 32 * kGradUnroll <= whole; b += 32 * kGradUnroll) {
        uint4 v[kGradUnroll];
        const int64_t at = (int64_t)(b + lane) * 16;
#pragma unroll
        for (int k = 0; k < kGradUnroll; ++k) v[k] = ld_stream(row + at + k * 512);
#pragma unroll
        for (int k = 0; k < kGradUnroll; ++k) {
            float x[8];
            grad_unit<kBf16, kEntropy, kFramed>(v[k], g, c, x);
            const int step = (b - chunk) / 32 + k;
            if (steps >> step & 1) {
                float y[8];
#pragma unroll
                for (int e = 0; e < per; ++e) y[e] = x[e];
                add_named<kBf16>(q, n_named, __shfl_sync(0xffffffffu, word, step), b + 32 * k, y);
#pragma unroll
                for (int e = 0; e < per; ++e) x[e] = y[e];
            }
            store_whole<kBf16>(out + at + k * 512, x);
        }
    }
    for (; b < stop; b += 32) {
        const uint4 v = load_unit<kBf16>(row, b + lane, stop, V);
        float x[8];
        grad_unit<kBf16, kEntropy, kFramed>(v, g, c, x);
        const int step = (b - chunk) / 32;
        if (steps >> step & 1) add_named<kBf16>(q, n_named, __shfl_sync(0xffffffffu, word, step), b, x);
        if (b + lane < stop) store_unit<kBf16>(out, b + lane, V, x);
    }
}

// A warp a piece, as in the forward pass; a lane reads a unit before it writes it, so the gradient may
// take the logits' place.
template <bool kBf16>
__global__ void __launch_bounds__(kVocabThreads, kGradBlocks) logprobs_grad_kernel(const LpGradArgs a) {
    constexpr int per = kBf16 ? 8 : 4;
    __shared__ Named named[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, V = a.rows.V;
    const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
    if (w >= a.rows.pieces) return;
    Named& q = named[warp];
    const int64_t start = piece_start(a.rows, w), end = piece_start(a.rows, w + 1);
    const float inv_T = 1.f / a.T;
    for (int64_t u = start; u < end;) {
        const int64_t r = u / a.rows.nvec, u0 = r * a.rows.nvec;
        const int c0 = (int)(u - u0), c1 = (int)(min(end, u0 + a.rows.nvec) - u0);
        const char* row = a.rows.base + r * a.rows.ld_bytes;
        char* out = a.out + r * a.out_bytes;
        u = u0 + c1;
        if (!in_bounds(r < a.rows.n_rows && c0 < c1 && c1 <= a.rows.nvec, a.status)) return;
        const float2 norm = a.norm[r];
        const bool empty = norm.y == 0.f;
        // named tokens and the sum of their gradients
        float pull = 0.f;
        int n_named = 0;
        __syncwarp();
        if (a.g_top) {
            n_named = a.top_k;
            for (int i = lane; i < a.top_k; i += 32) {
                int id = a.top_ids[r * a.top_k + i];
                float g = a.g_top[r * a.top_k + i];
                if (id >= V) report(a.status, ESTP_ERR_INVALID_ARG);
                if (id < 0 || id >= V || empty) {
                    id = -1;
                    g = 0.f;
                }
                q.id[i] = id;
                q.g[i] = g * inv_T;
                pull += g;
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) pull += __shfl_xor_sync(0xffffffffu, pull, off);
        }
        if (a.g_logprob) {
            int id = a.targets[r];
            float g = a.g_logprob[r];
            if (id >= V && lane == 0) report(a.status, ESTP_ERR_INVALID_ARG);
            if (id < 0 || id >= V || empty) {
                id = -1;
                g = 0.f;
            }
            if (lane == 0) {
                q.id[n_named] = id;
                q.g[n_named] = g * inv_T;
            }
            ++n_named;
            pull += g;
        }
        __syncwarp();
        const float gH = a.g_entropy && !empty ? a.g_entropy[r] : 0.f, gl = a.g_lse ? a.g_lse[r] : 0.f;
        // nothing for the row as a whole: zeros, whatever its logits hold
        const bool flat = empty || (gl - pull == 0.f && gH == 0.f);
        RowGrad g{pivot(norm.x), 0.f, 0.f, 0.f, false};
        g.M = g.m * a.c;
        g.framed = near_frame(g.M);
        if (!flat) {
            const float f = inv_T / norm.y, off = frame_off(g.m, a.c), back = ex2(-off);
            g.B = -f * gH * kLn2 * back;
            g.A = f * (gl - pull + (gH != 0.f ? gH * (logf(norm.y) - a.entropy[r]) : 0.f)) * back - g.B * off;
        }
        for (int chunk = c0; chunk < c1; chunk += 1024) {
            // the units of this chunk with a named token, lane l's word those of its step l
            bool any = false;
            for (int i = lane; i < n_named; i += 32) any |= q.id[i] >= 0 && (unsigned)(q.id[i] / per - chunk) < 1024u;
            uint32_t word = 0, steps = 0;
            if (__any_sync(0xffffffffu, any)) {
                q.bits[lane] = 0;
                __syncwarp();
                for (int i = lane; i < n_named; i += 32) {
                    const unsigned k = (unsigned)(q.id[i] / per - chunk);
                    if (q.id[i] >= 0 && k < 1024u) atomicOr(&q.bits[k >> 5], 1u << (k & 31));
                }
                __syncwarp();
                word = q.bits[lane];
                steps = __ballot_sync(0xffffffffu, word != 0);
                __syncwarp();
            }
            const int stop = min(c1, chunk + 1024);
            if (flat) {
                for (int b = chunk; b < stop; b += 32) {
                    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    const int step = (b - chunk) / 32;
                    if (steps >> step & 1) add_named<kBf16>(q, n_named, __shfl_sync(0xffffffffu, word, step), b, x);
                    if (b + lane < stop) store_unit<kBf16>(out, b + lane, V, x);
                }
            } else if (!g.framed) {
                grad_chunk<kBf16, true, false>(row, out, chunk, stop, V, g, a.c, q, n_named, word, steps);
            } else if (gH != 0.f) {
                grad_chunk<kBf16, true, true>(row, out, chunk, stop, V, g, a.c, q, n_named, word, steps);
            } else {
                grad_chunk<kBf16, false, true>(row, out, chunk, stop, V, g, a.c, q, n_named, word, steps);
            }
        }
    }
}

}  // namespace

estp_status launch_token_logprobs(estp_ctx* ctx, const void* logits, estp_dtype dtype, int64_t n_rows, int64_t V,
                                  int64_t ld, const int32_t* targets, float T, int top_k, float* logprob,
                                  float* entropy, float* norm, int32_t* top_ids, float* top_logprobs,
                                  cudaStream_t st) {
    LpArgs a;
    a.rows = vocab_rows(ctx, logits, dtype, n_rows, V, ld, 32 * kVocabUnroll, kVocabBlocks);
    a.targets = targets;
    a.T = T;
    a.c = (float)(1.4426950408889634 / (double)T);
    a.top_k = top_k;
    a.logprob = logprob;
    a.entropy = entropy;
    a.norm = reinterpret_cast<float2*>(norm);
    a.top_ids = top_ids;
    a.top_logprobs = top_logprobs;
    a.part = ctx->vocab_part;
    a.lists = ctx->vocab_lists;
    a.status = ctx->status;
    const cudaError_t e = dtype == ESTP_BF16 ? launch_forward<true>(a, st) : launch_forward<false>(a, st);
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "log probability launch");
}

estp_status launch_token_logprobs_grad(estp_ctx* ctx, const void* logits, estp_dtype dtype, int64_t n_rows, int64_t V,
                                       int64_t ld, const float* norm, const float* entropy, const int32_t* targets,
                                       float T, int top_k, const int32_t* top_ids, const float* g_logprob,
                                       const float* g_entropy, const float* g_lse, const float* g_top, void* out,
                                       int64_t ld_out, cudaStream_t st) {
    LpGradArgs a;
    a.rows = vocab_rows(ctx, logits, dtype, n_rows, V, ld, 32 * kGradUnroll, kGradBlocks);
    a.out = static_cast<char*>(out);
    a.out_bytes = ld_out * esize(dtype);
    a.norm = reinterpret_cast<const float2*>(norm);
    a.entropy = entropy;
    a.targets = targets;
    a.top_ids = top_ids;
    a.g_logprob = g_logprob;
    a.g_entropy = g_entropy;
    a.g_lse = g_lse;
    a.g_top = g_top;
    a.T = T;
    a.c = (float)(1.4426950408889634 / (double)T);
    a.top_k = top_k;
    a.status = ctx->status;
    const unsigned blocks = (unsigned)((a.rows.pieces + kWarps - 1) / kWarps);
    if (dtype == ESTP_BF16) logprobs_grad_kernel<true><<<blocks, kVocabThreads, 0, st>>>(a);
    else logprobs_grad_kernel<false><<<blocks, kVocabThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "log probability gradient launch");
}

}  // namespace estp
