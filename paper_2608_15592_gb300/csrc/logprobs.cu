// Log probabilities of given tokens with the row's entropy and its greatest alternatives, and the
// gradient of all of them with respect to the logits.
//
// logprobs_kernel streams the logits once: a warp takes one of the equal pieces of the flat run of
// 16-byte units (vocab.cuh), keeps (m, s, t) per lane and, where alternatives are asked for, the
// list of the 32 R greatest logits it has met.  A row that lies within a piece is finished by its warp; of a
// row cut between warps each writes its part, and the warp that writes a row's last part joins all of them, in an
// order that does not depend on which it is.  Where rows are few, logprobs_few_kernel gives each a number of blocks,
// whose warps join their parts in shared memory first.
//
// Bound: the read of the logits.  42 instructions and 8 exponentials for 256 bf16 logits leave the issue slots half idle
// at the memory's rate: 4096 rows of 128256 tokens in 159 us (6.6 TB/s), 2048 of 152064 in 103; some 14 us of a call are
// its launch, the first loads and the last row's join, which is what 1024 rows (60 us for 46 us of bytes) and less pay.
// A batch that holds a mask is summed twice (vocab.cuh): with half of all tokens masked the 4096 rows take 217.
// Alternatives add what their candidates take: 1537 rows of 152064 in 123 us with 64, 44 % of the instructions for
// the lists, in chains that five warps a scheduler issue at 2.1 a clock.  Measured beside it: bounds not shared between the
// warps of a row 133; candidates kept in no order and thinned out by the bits of their keys 127; the next batch copied into shared
// memory meanwhile 140 and four blocks an SM with four loads 142 (both take more instructions).  20 alternatives take 104, 128
// take 156: the kernel for more than 64 spills.
//
// The list.  A candidate is a 64-bit key: the logit's bits in the order of the numbers above the token's
// index, inverted; so keys are unique, a greater key is a greater logit or the same one at a lower
// index, and whatever order candidates come in, the result is one.  A warp compares the maximum of each
// batch with a bound below which nothing can enter; only units above it are looked at, and what
// passes goes to a buffer in shared memory, which is sorted and merged into the list when
// it holds 32 R candidates.  The bound starts as a logit that at least top_k of the first batch's
// partial maxima reach, and after each merge is the next number above the list's entry top_k (later
// tokens have higher indices: equals lose), or what the warps on the same row have all reached in part (post).  Of n logits
// about top_k ln(n / top_k) pass.
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
// The steps j, j / 2, .. 1 of a bitonic network: keys i and i ^ j, the greater one to the lower index
// where bit `size` of i is clear.  (Loops, not unrolled: this code runs seldom, between code that
// should stay in the instruction cache.)
template <int R>
__device__ __forceinline__ void exchanges(uint64_t (&x)[R], int size, int j, int lane) {
#pragma unroll
    for (int w = R / 2; w > 0; w /= 2)
        if (32 * w <= j) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if ((r & w) == 0) {
                    const bool down = (r * 32 & size) != 0;
                    const uint64_t a = x[r], b = x[r | w];
                    if ((a < b) != down) {
                        x[r] = b;
                        x[r | w] = a;
                    }
                }
        }
#pragma unroll 1
    for (j = j < 16 ? j : 16; j > 0; j >>= 1) {
        const bool low = (lane & j) == 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint64_t y = __shfl_xor_sync(0xffffffffu, x[r], j);
            const bool up = (((r * 32 + lane) & size) == 0) == low;
            x[r] = (x[r] > y) == up ? x[r] : y;
        }
    }
}

template <int R>
__device__ __forceinline__ void sort_keys(uint64_t (&x)[R], int lane) {
#pragma unroll 1
    for (int size = 2; size <= 32 * R; size *= 2) exchanges<R>(x, size, size / 2, lane);
}

// The greatest 32 R of two descending lists, descending.
template <int R>
__device__ __forceinline__ void merge_keys(uint64_t (&x)[R], const uint64_t (&y)[R], int lane) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint64_t o = __shfl_sync(0xffffffffu, y[R - 1 - r], 31 - lane);
        x[r] = x[r] > o ? x[r] : o;
    }
    exchanges<R>(x, 64 * R, 16 * R, lane);
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
    uint32_t units[32 + 32 * kVocabUnroll];  // a batch adds up to 32 kVocabUnroll; they are taken by 32
    int count, n_units;
    int first_mate, mates, each;  // warps that stream this row too, itself among them, from this one; 1: none
    uint32_t row;                 // (+ 1)
    volatile uint64_t posted;     // a row (+ 1) above the ordered bits of a logit that `each` of the warp's tokens reach
};

// What the warps of a block that stream the same row tell each other.  A logit that `each` tokens of each of the `mates`
// reach is reached by mates x each >= top_k tokens of the row: smaller ones cannot be alternatives, whatever the
// warps still meet.  What is posted is read as it comes, which changes how much is looked at and not what is found.
template <int R>
__device__ __forceinline__ void post(Candidates<R>* q, uint32_t bits) {
    const uint64_t x = (uint64_t)q->row << 32 | bits;  // (a warp's rows ascend)
    if ((threadIdx.x & 31) == 0 && x > q->posted) q->posted = x;
}
template <int R>
__device__ __forceinline__ float shared_bound(const Candidates<R>* q) {
    const int lane = threadIdx.x & 31;
    uint32_t bits = 0xFFFFFFFFu;
    if (lane < q->mates) {
        const uint64_t x = (q + q->first_mate + lane)->posted;
        bits = (uint32_t)(x >> 32) == q->row ? (uint32_t)x : 0u;
    }
    bits = __reduce_min_sync(0xffffffffu, bits);
    return bits > 0x007FFFFFu ? unordered(bits) : -INFINITY;
}

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

// Looks at the units that wait (from the segment's first one, c0, on), one a lane (their second read comes from
// L2): whole 32s of them or all.  Candidates are at least `floor`; returns the bound for the tokens that follow.
template <bool kBf16, int R>
__device__ __noinline__ float take_units(Candidates<R>* q, const char* row, int c0, int limit, int top_k, float floor,
                                         bool all, int* status) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31;
    int n = q->n_units;
    // these units are not in the order of the tokens: an equal of the list's last may come before it or after
    uint64_t last = q->list[top_k - 1];
    float cut = last ? fmaxf(floor, key_logit(last)) : floor;
    while (n >= 32 || (all && n > 0)) {
        const int take = n < 32 ? n : 32;
        n -= take;
        if (lane < take) {
            const int c = c0 + (int)q->units[n + lane], first = c * per;
            if (first < limit) {
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
            if (q->mates > 1) {
                if (const uint64_t x = q->list[q->each - 1]) post<R>(q, (uint32_t)(x >> 32));
                floor = fmaxf(floor, shared_bound<R>(q));
            }
            cut = fmaxf(floor, last ? key_logit(last) : floor);
        }
        __syncwarp();
    }
    if (lane == 0) q->n_units = n;
    __syncwarp();
    return last ? fmaxf(floor, unordered((uint32_t)(last >> 32) + 1)) : floor;  // the next number above it
}

// The lists of a block's warps merged into the first one's, by pairs (the whole block).
template <int R>
__device__ __forceinline__ void merge_block(Candidates<R>* cand) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll 1
    for (int half = kWarps / 2; half > 0; half /= 2) {
        if (warp < half) merge_lists<R>(cand[warp].list, cand[warp + half].list, lane);
        __syncthreads();
    }
}

// Masked tokens (-inf) do not become candidates: a list that is short of top_k keys has every token that is not masked,
// and write_row fills it up.
constexpr float kLowest = -3.4028234663852886e38f;

// A logit that at least top_k of the warp's 32 G values reach and hardly more (or -inf): the order bits from the first one
// down in which the values differ, as far as 16 of them go.  `shared`: the ordered bits of the greatest logit met on the
// way that `each` <= top_k of them reach.
template <int G>
__device__ __forceinline__ float reached_by(const float (&x)[G], int top_k, int each, uint32_t& shared) {
    uint32_t o[G], lo = 0xFFFFFFFFu, hi = 0;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        o[g] = ordered(x[g]);
        lo = min(lo, o[g]);
        hi = max(hi, o[g]);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    shared = 0;
    int bit = 31 - __clz(lo ^ hi);  // -1: all alike
    uint32_t t = bit < 0 ? hi : hi & ~((2u << bit) - 1);
#pragma unroll 1
    for (; bit >= 16; --bit) {
        const uint32_t next = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int g = 0; g < G; ++g) n += __popc(__ballot_sync(0xffffffffu, o[g] >= next));
        if (n >= top_k) {
            t = next;
            if (n <= top_k + top_k / 8) break;
        } else if (n >= each) {
            shared = max(shared, next);
        }
    }
    shared = max(shared, t);
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
    int blocks, span;  // few rows: blocks a row and units a warp (0: equal pieces)
    float4* part;      // [slots]: m, s, t of a part: two a piece, for its first and its last row, or one a block
    uint64_t* lists;   // [slots][32 R]
    uint32_t* count;   // [slots]: parts that have arrived of a row, by its first piece or its index
    int64_t slots;
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
    float floor = -INFINITY, bound = -INFINITY;
    for (int b = c0; b < c1; b += 32 * kVocabUnroll) {
        if (R > 0) fetch_units(row, b + 32 * kVocabUnroll, 32 * kVocabUnroll, c1);  // (the lists' work hides it: 129 -> 126 us)
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
        const UnitMaxima<kBf16, kVocabUnroll> um(v);
        const float bm = um.all();
        if constexpr (R > 0) {
            if (b == c0) {
                constexpr int G = 2 * R, w = kVocabUnroll / G;  // 64 R maxima
                float g[G];
#pragma unroll
                for (int i = 0; i < G; ++i) g[i] = units_max<kBf16, w>(v + i * w);
                uint32_t shared;
                floor = bound = fmaxf(reached_by<G>(g, a.top_k, q->each, shared), kLowest);
                if (q->mates > 1) post<R>(q, shared);
            } else if (q->mates > 1) {
                floor = fmaxf(floor, shared_bound<R>(q));
                bound = fmaxf(bound, floor);
            }
            // units with candidates are queued; the longer part waits until the batch is in the sums
            if (__any_sync(0xffffffffu, bm >= bound)) {
                uint32_t hits = um.reached(bound);
                if (hits)
                    for (int at = atomicAdd(&q->n_units, __popc(hits)); hits; hits &= hits - 1, ++at)
                        if (in_bounds(at < 32 + 32 * kVocabUnroll, a.status)) q->units[at] = (uint32_t)(c - c0 + 32 * (__ffs(hits) - 1));
                __syncwarp();
            }
        }
        st.template add_units<kBf16>(v, bm, a.c);
        if constexpr (R > 0) {
            if (q->n_units >= 32) bound = take_units<kBf16, R>(q, row, c0, limit, a.top_k, floor, false, a.status);
            __syncwarp();
        }
    }
    if constexpr (R > 0) {
        take_units<kBf16, R>(q, row, c0, limit, a.top_k, floor, true, a.status);
        take_waiting<R>(q, a.top_k, true);
    }
    return st.row(a.c);
}

// A row's target and the bits of its logit (lane 0): the one asked for where the row begins, the other, which needs it,
// behind the stream.
struct Target {
    int t;
    uint32_t z;
};

__device__ __forceinline__ Target ask_target(const LpArgs& a, int64_t r) {
    Target x{-1, 0u};
    if (a.logprob && (threadIdx.x & 31) == 0 && in_bounds(r < a.rows.n_rows, a.status)) x.t = a.targets[r];
    return x;
}

template <bool kBf16>
__device__ __forceinline__ void ask_logit(const LpArgs& a, const char* row, Target& x) {
    if (x.t >= 0 && x.t < a.rows.V)
        x.z = kBf16 ? (uint32_t)reinterpret_cast<const uint16_t*>(row)[x.t] : reinterpret_cast<const uint32_t*>(row)[x.t];
}

// (z - m) / T by halves: the distance of two finite logits may overflow where its quotient does not.
__device__ __forceinline__ float below(float z, float m, float T) { return (0.5f * z - 0.5f * m) / T * 2.f; }

// What a row's statistics and list say, written by a warp.
template <bool kBf16, int R>
__device__ __forceinline__ void write_row(const LpArgs& a, int64_t r, const Target& x, const RowStat& st,
                                          const uint64_t* list) {
    const int lane = threadIdx.x & 31;
    if (!in_bounds(r >= 0 && r < a.rows.n_rows, a.status)) return;
    const bool empty = st.s == 0.f;  // (NaN is not)
    const float ls = empty ? 0.f : logf(st.s), m = pivot(st.m);
    if (lane == 0) {
        if (a.entropy) a.entropy[r] = empty ? 0.f : ls - kLn2 * (st.t / st.s);
        if (a.norm) a.norm[r] = make_float2(st.m, st.s);
        if (a.logprob) {
            float lp = x.t < 0 ? 0.f : below(__uint_as_float(kBf16 ? x.z << 16 : x.z), m, a.T) - ls;
            if (x.t >= a.rows.V) {
                report(a.status, ESTP_ERR_INVALID_ARG);
                lp = NAN;
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
                if (k == 0 && !none) continue;
                a.top_ids[r * a.top_k + i] = none ? -1 : key_token(k);
                if (a.top_logprobs) a.top_logprobs[r * a.top_k + i] = none ? NAN : below(key_logit(k), m, a.T) - ls;
            }
        if (list[a.top_k - 1] == 0 && !none) {
            // short of tokens: the masked ones of lowest index follow, which are among the first top_k
            int n = 0;
            while (n < a.top_k && list[n] != 0) ++n;
            const int have = n;
            for (int v0 = 0; v0 < a.top_k && n < a.top_k; v0 += 32) {
                const int v = v0 + lane;
                bool masked = v < a.top_k;
                for (int i = 0; i < have; ++i) masked &= key_token(list[i]) != v;
                const uint32_t all = __ballot_sync(0xffffffffu, masked);
                const int at = n + __popc(all & ((1u << lane) - 1));
                if (masked && at < a.top_k) {
                    a.top_ids[r * a.top_k + at] = v;
                    if (a.top_logprobs) a.top_logprobs[r * a.top_k + at] = -INFINITY;
                }
                n += __popc(all);
            }
        }
    }
}

// A part of a row goes to its slot (a warp).
template <int R>
__device__ __forceinline__ void put_part(const LpArgs& a, int64_t slot, const RowStat& st, const uint64_t* list) {
    const int lane = threadIdx.x & 31;
    if (!in_bounds(slot >= 0 && slot < a.slots, a.status)) return;
    if (lane == 0) a.part[slot] = make_float4(st.m, st.s, st.t, 0.f);
    if constexpr (R > 0)
        for (int i = lane; i < 32 * R; i += 32) a.lists[slot * (32 * R) + i] = list[i];
}

// The statistics of a row's n parts, part 0 in `slot0` and the others from `slot` on, `step` apart: joined in one
// order whichever warp does it.
__device__ __forceinline__ RowStat join_parts(const LpArgs& a, int64_t slot0, int64_t slot, int step, int n) {
    RowStat st = no_stat();
    for (int i = threadIdx.x & 31; i < n; i += 32) {
        const int64_t at = i ? slot + (int64_t)(i - 1) * step : slot0;
        if (!in_bounds(at >= 0 && at < a.slots, a.status)) break;
        const float4 x = __ldcg(&a.part[at]);
        join(st, RowStat{x.x, x.y, x.z}, a.c);
    }
    __syncwarp();
    join_lanes(st, a.c);
    return st;
}

// The lists of parts i0, i0 + by, .. merged into `list` (keys all differ: any order gives the same).
template <int R>
__device__ __forceinline__ void merge_parts(const LpArgs& a, int64_t slot0, int64_t slot, int step, int n, int i0, int by,
                                            uint64_t* list) {
    const int lane = threadIdx.x & 31;
    uint64_t x[R], y[R];
#pragma unroll
    for (int k = 0; k < R; ++k) x[k] = y[k] = 0;
#pragma unroll 1
    for (int i = i0; i < n + by; i += by) {  // the next part loads while this one is merged
        uint64_t z[R];
        const int64_t at = (i ? slot + (int64_t)(i - 1) * step : slot0) * (32 * R);
#pragma unroll
        for (int k = 0; k < R; ++k) z[k] = i < n && in_bounds(at >= 0 && at < a.slots * (32 * R), a.status) ? __ldcg(&a.lists[at + k * 32 + lane]) : 0;
        if (i > i0) merge_keys<R>(x, y, lane);
#pragma unroll
        for (int k = 0; k < R; ++k) y[k] = z[k];
    }
#pragma unroll
    for (int k = 0; k < R; ++k) list[k * 32 + lane] = x[k];
    __syncwarp();
}

template <int R>
__device__ __forceinline__ void clear_list(Candidates<R>* q, uint32_t row, int first_mate, int mates, int top_k) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
    for (int i = lane; i < 32 * R; i += 32) q->list[i] = 0;
    if (lane == 0) {
        q->count = q->n_units = 0;
        q->row = row;
        q->first_mate = first_mate;
        q->mates = mates;
        q->each = (top_k + mates - 1) / mates;
    }
    __syncwarp();
}

// Many rows: a warp an equal piece of the flat run.
template <bool kBf16, int R>
__global__ void __launch_bounds__(kVocabThreads, kVocabBlocks) logprobs_kernel(const LpArgs a) {
    constexpr int kLists = R ? R : 1;
    __shared__ Candidates<kLists> cand[R ? kWarps : 1];
    const int warp = threadIdx.x >> 5;
    const int64_t first = (int64_t)blockIdx.x * kWarps, w = first + warp;
    if constexpr (R > 0) {
        if (threadIdx.x < kWarps) cand[threadIdx.x].posted = 0;
        __syncthreads();
    }
    if (w >= a.rows.pieces) return;
    Candidates<kLists>* q = R ? &cand[warp] : nullptr;
    const int64_t start = piece_start(a.rows, w), end = piece_start(a.rows, w + 1);
    for (int64_t u = start; u < end;) {
        const int64_t r = quotient(u, a.rows.nvec), u0 = r * a.rows.nvec;
        const int c0 = (int)(u - u0), c1 = (int)(min(end, u0 + a.rows.nvec) - u0);
        const char* row = a.rows.base + r * a.rows.ld_bytes;
        if (!in_bounds(r < a.rows.n_rows && c0 < c1 && c1 <= a.rows.nvec, a.status)) return;
        Target x = ask_target(a, r);
        RowStat st;
        if constexpr (R > 0) {
            int mate = warp, mates = 1;
            if (c0 != 0 || c1 != a.rows.nvec) {
                const int64_t lo = piece_of(a.rows, u0) - first, hi = piece_of(a.rows, u0 + a.rows.nvec - 1) - first;
                mate = lo > 0 ? (int)lo : 0;
                mates = (int)(hi < kWarps - 1 ? hi : kWarps - 1) - mate + 1;
            }
            clear_list<R>(q, (uint32_t)r + 1, mate - warp, mates, a.top_k);
            st = stream_row<kBf16, R>(a, row, c0, c1, q);
        } else {
            st = stream_row<kBf16, 0>(a, row, c0, c1, nullptr);
        }
        if (R == 0) fetch_next(a.rows, row, u0 + c1, end);
        ask_logit<kBf16>(a, row, x);
        join_lanes(st, a.c);
        bool write = true;
        if (c0 != 0 || c1 != a.rows.nvec) {
            put_part<R>(a, w * 2 + (u == start ? 0 : 1), st, R ? q->list : nullptr);
            // the row's pieces lo .. hi; only the first may begin in the row before it
            const int64_t lo = piece_of(a.rows, u0), hi = piece_of(a.rows, u0 + a.rows.nvec - 1);
            const int64_t slot0 = lo * 2 + (piece_start(a.rows, lo) < u0 ? 1 : 0);
            const int n = (int)(hi - lo + 1);
            write = in_bounds(lo >= 0 && lo < a.slots, a.status) && arrive(a.count + lo, n);
            if (write) {
                st = join_parts(a, slot0, lo * 2 + 2, 2, n);
                if constexpr (R > 0) merge_parts<R>(a, slot0, lo * 2 + 2, 2, n, 0, 1, q->list);
            }
        }
        if (write) write_row<kBf16, R>(a, r, x, st, R ? q->list : nullptr);
        u = u0 + c1;
    }
}

// Few rows: a.blocks blocks a row, whose warps join their parts themselves.
template <bool kBf16, int R>
__global__ void __launch_bounds__(kVocabThreads, kVocabBlocks) logprobs_few_kernel(const LpArgs a) {
    constexpr int kLists = R ? R : 1;
    __shared__ Candidates<kLists> cand[R ? kWarps : 1];
    __shared__ RowStat stats[kWarps];
    __shared__ int last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = blockIdx.x / a.blocks, b = blockIdx.x - r * a.blocks;
    const char* row = a.rows.base + r * a.rows.ld_bytes;
    Candidates<kLists>* q = R ? &cand[warp] : nullptr;
    Target x{-1, 0u};
    if (warp == 0) x = ask_target(a, r);
    const int c0 = min(a.rows.nvec, (b * kWarps + warp) * a.span), c1 = min(a.rows.nvec, c0 + a.span);
    RowStat st = no_stat();
    const bool some = c0 < c1 && in_bounds(r < a.rows.n_rows && c1 <= a.rows.nvec, a.status);
    if constexpr (R > 0) {
        clear_list<R>(q, 1, 0, 1, a.top_k);
        if (some) st = stream_row<kBf16, R>(a, row, c0, c1, q);
    } else {
        if (some) st = stream_row<kBf16, 0>(a, row, c0, c1, nullptr);
    }
    ask_logit<kBf16>(a, row, x);
    join_lanes(st, a.c);
    if (lane == 0) stats[warp] = st;
    __syncthreads();
    if constexpr (R > 0) merge_block<R>(cand);
    const int64_t slot = (int64_t)r * a.blocks;
    if (warp == 0) {
        st = lane < kWarps ? stats[lane] : no_stat();
        join_lanes(st, a.c);
        bool l = false;
        if (a.blocks > 1) {
            put_part<R>(a, blockIdx.x, st, R ? q->list : nullptr);
            l = in_bounds(r < a.slots, a.status) && arrive(a.count + r, a.blocks);
        } else {
            write_row<kBf16, R>(a, r, x, st, R ? q->list : nullptr);
        }
        if (lane == 0) last = l;
    }
    if (a.blocks == 1) return;
    __syncthreads();
    if (!last) return;
    if constexpr (R > 0) {
        merge_parts<R>(a, slot, slot + 1, 1, a.blocks, warp, kWarps, q->list);
        __syncthreads();
        merge_block<R>(cand);
    }
    if (warp == 0) write_row<kBf16, R>(a, r, x, join_parts(a, slot, slot + 1, 1, a.blocks), R ? q->list : nullptr);
}

template <bool kBf16, int R>
cudaError_t launch_forward(const LpArgs& a, cudaStream_t st) {
    if (a.blocks) logprobs_few_kernel<kBf16, R><<<(unsigned)(a.rows.n_rows * a.blocks), kVocabThreads, 0, st>>>(a);
    else logprobs_kernel<kBf16, R><<<(unsigned)((a.rows.pieces + kWarps - 1) / kWarps), kVocabThreads, 0, st>>>(a);
    return cudaGetLastError();
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

constexpr int kGradUnroll = 4, kGradBlocks = 3;

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
        for (int k = 0; k < kGradUnroll; ++k) v[k] = ld_once(row + at + k * 512);
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
//
// Bound: the read and the write.  4096 rows of 128256 tokens in 331 to 341 us (6.2 TB/s of both and more); a kernel that only reads
// and writes takes 323 to 343 with as many warps and loads.  Three blocks an SM of four loads a lane: 335, four blocks 341, two
// of eight loads 333 but 26 instead of 23 for 501 fp32 rows of 32001.
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
        const int64_t r = quotient(u, a.rows.nvec), u0 = r * a.rows.nvec;
        const int c0 = (int)(u - u0), c1 = (int)(min(end, u0 + a.rows.nvec) - u0);
        const char* row = a.rows.base + r * a.rows.ld_bytes;
        char* out = a.out + r * a.out_bytes;
        u = u0 + c1;
        if (!in_bounds(r < a.rows.n_rows && c0 < c1 && c1 <= a.rows.nvec, a.status)) return;
        const float2 norm = a.norm[r];
        const bool empty = norm.y == 0.f;
        // named tokens and the sum of their gradients
        float pull = 0.f;
        bool asked = false;  // something of the row at all
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
                asked |= g != 0.f;
            }
            asked = __any_sync(0xffffffffu, asked);
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
            asked |= g != 0.f;
        }
        __syncwarp();
        const float gH = a.g_entropy && !empty ? a.g_entropy[r] : 0.f, gl = a.g_lse ? a.g_lse[r] : 0.f;
        // nothing for the row as a whole: zeros but for named tokens, and where nothing is asked whatever its logits hold
        // (in a row of NaN what cancels is NaN)
        asked |= gl != 0.f;
        const bool flat = empty || (gl - pull == 0.f && gH == 0.f && !(asked && isnan(norm.y)));
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
    const int64_t most = (int64_t)ctx->num_sms * kVocabBlocks;  // blocks at once
    a.slots = 2 * most * kWarps;
    a.blocks = a.span = 0;
    if (n_rows <= most / 2) {
        // Blocks a row: two for every place on the GPU between all rows, a batch a warp at least.  One row of 152064
        // tokens with 20 alternatives takes 11.5 us, by equal pieces and a second launch that joined them 19.
        const int64_t batches = ((int64_t)a.rows.nvec + kWarps * 32 * kVocabUnroll - 1) / (kWarps * 32 * kVocabUnroll);
        const int64_t want = 2 * most / n_rows;
        a.blocks = (int)(batches < want ? batches : want);
        a.span = (a.rows.nvec + a.blocks * kWarps - 1) / (a.blocks * kWarps);
    } else if (top_k > 0 && a.rows.pieces > n_rows) {
        // a list costs as much to begin as some thousand logits: pieces of whole rows while that idles few warps (fewer
        // than 16 a row here, and a row has at most 2^24 units)
        const int64_t per_row = a.rows.pieces / n_rows;
        if (4 * per_row * n_rows >= 3 * a.rows.pieces) cut_rows(a.rows, per_row * n_rows, (int)per_row);
    }
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
    a.count = ctx->vocab_count;
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
