// Distillation from a teacher of whom each row's top logits are known: the divergence of the student's
// distribution from the teacher's, and its gradient with respect to the student's logits.
//
// With the named tokens id_j, the teacher's q_j over them, q_r what it leaves to all others (0 without
// the tail), Q = sum q_j and p the student's softmax at temperature T, p_r = sum of p over the others:
//   L = sum_j q_j (ln q_j - ln p_id_j) + q_r (ln q_r - ln p_r)
//   T dL/dz_v = (Q + q_r) p_v - q_j            for a named token
//             = (Q + q_r) p_v - q_r p_v / p_r  for another one
// p_r is summed over the other tokens themselves and not formed as 1 - sum p_id, which would lose it
// where the named tokens hold nearly everything; the sum has a maximum of its own, so it does not
// underflow beside a named token far above.
//
// Bound: one read and one write of the row.  The gradient needs the row's sum before its first element, so a row is
// either read twice or kept.  It is kept: a cluster of C CTAs takes a row, each a slice that fits its shared memory beside
// those of the other CTAs of the SM.  Rows too long for that are read twice (distill_long_kernel), very short ones from the
// caches (distill_short_kernel); the loss alone is one read (distill_eval_kernel).
//
// 2048 rows of 128256 bf16 tokens take 177 us (155 at the copy's rate; a block a row with both passes from memory: 419), 1021
// of 152064 with the tail 128 (92).  Two exponentials a logit and some 110 instructions for 256 of them are issued at
// 2.2 a clock of 4: what is left is their latency where warps wait for the row's barrier.
#include <type_traits>

#include "split_rules.cuh"
#include "vocab.cuh"

namespace estp {
namespace {

constexpr int kK = kMaxAlternatives;

// Sums of two floats (some 48 bits): a + b and a b exactly, and a + b of such.
struct Two {
    float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return Two{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two two_prod(float a, float b) {
    const float p = __fmul_rn(a, b);
    return Two{p, __fmaf_rn(a, b, -p)};
}
__device__ __forceinline__ Two plus(Two a, Two b) {
    const Two s = two_sum(a.hi, b.hi);
    return Two{s.hi, s.lo + (a.lo + b.lo)};
}
__device__ __forceinline__ Two times(Two a, Two b) {
    const Two p = two_prod(a.hi, b.hi);
    return Two{p.hi, p.lo + (a.hi * b.lo + a.lo * b.hi)};
}

struct DistillArgs {
    const char* base;
    int64_t ld_bytes;
    int64_t n_rows;
    int32_t V, nvec;
    const int32_t* ids;
    const float* teacher;
    int K, tail;
    float T, c;
    Two inv_T;  // 1 / T
    const float* weight;
    float* loss;
    char* out;
    int64_t out_bytes;
    int* status;
};

// Units [u0, u1) of row r are the logits' and the gradient's; with `whole` none of them is the row's partial last one.
__device__ __forceinline__ bool units_there(const DistillArgs& a, int64_t r, int u0, int u1, int per, bool whole) {
    return in_bounds(r >= 0 && r < a.n_rows && u0 >= 0 && u0 < u1 && (whole ? u1 <= a.V / per : u1 <= a.nvec), a.status);
}

__device__ __forceinline__ void put_loss(const DistillArgs& a, int64_t r, float loss) {
    if ((threadIdx.x & 31) == 0 && in_bounds(r >= 0 && r < a.n_rows, a.status)) a.loss[r] = loss;
}

// The teacher's side of a row, which its logits have no part in but for those of the named tokens.
struct Teacher {
    int32_t id[kK];            // -1: none
    float lq[kK], q[kK], z[kK];  // ln q, q, the student's logit
    RowStat in;                // with the tail: statistics of the named tokens
    float Q, rest, g;          // the sum of the q, 1 less it, row weight / T
    float Q_lo, rest_lo;       // what the first two were rounded by
    int some, repeated;        // has entries; has a token twice
};

// What every element of a row's gradient takes from its sums.
struct Factors {
    float m, s;      // maximum and sum of all tokens
    float pivot, A;  // an element that is not named: A 2^((z - pivot) c)
    float M, near;   // where pivot has a near frame: near 2^(z c - M)
    bool framed;
    float rest;
    bool empty, zero;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
    return x;
}

// A row's entries, four a lane (entry 32 i + lane), on their way into Teacher: tokens and values first, then the
// student's logits, which need the tokens' addresses.  Each is asked for a row before it is used.
constexpr int kPer = kK / 32;
struct Entries {
    int32_t id[kPer];
    uint32_t z[kPer];  // bits as loaded: a conversion would wait for them
    float x[kPer], w;
    bool repeated;
};

// What a row's entries are copied to first (asked for two rows ahead).
struct Asked {
    int32_t id[kK];
    float x[kK], w;
};

__device__ __forceinline__ void copy_word(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ void ask_entries(const DistillArgs& a, int64_t r, Asked& q) {
    if (r >= a.n_rows) return;
    const int lane = threadIdx.x & 31;
    for (int j = lane; j < a.K; j += 32) {
        const int64_t at = r * a.K + j;
        if (!in_bounds(at < a.n_rows * a.K, a.status)) continue;
        copy_word(&q.id[j], a.ids + at);
        copy_word(&q.x[j], a.teacher + at);
    }
    if (lane == 0 && a.weight) copy_word(&q.w, a.weight + r);
}

__device__ __forceinline__ void take_entries(const DistillArgs& a, const Asked& q, Entries& e) {
    const int lane = threadIdx.x & 31;
    copies_done();
    __syncwarp();
    e.w = a.weight ? q.w : 1.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {  // (here and below, what lies past K costs a branch)
        const int j = i * 32 + lane;
        e.id[i] = -1;
        e.x[i] = -INFINITY;
        if (i * 32 < a.K && j < a.K) {
            e.id[i] = q.id[j];
            e.x[i] = q.x[j];
        }
    }
    __syncwarp();
}

// Tokens outside of the vocabulary are left out; repeated ones are found by a table of kSlots places with linear
// probing, empty (-1) before and after.  Then the logits are asked for.
constexpr int kSlots = 256;
template <bool kBf16>
__device__ __forceinline__ void check_entries(const DistillArgs& a, int64_t r, Entries& e, int32_t* table) {
    const int lane = threadIdx.x & 31;
    uint32_t slot[kPer];
    int old[kPer];
    bool bad = false, again = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        old[i] = -1;
        if (i * 32 >= a.K) continue;
        if (e.id[i] >= a.V) {
            bad = true;
            e.id[i] = -1;
        }
        slot[i] = (uint32_t)e.id[i] * 2654435761u >> 24;
        old[i] = e.id[i] >= 0 ? atomicCAS(&table[slot[i]], -1, e.id[i]) : -1;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (i * 32 >= a.K) continue;
        for (int tries = 1; tries < kSlots && old[i] != -1 && old[i] != e.id[i]; ++tries) {
            slot[i] = (slot[i] + 1) % kSlots;
            old[i] = atomicCAS(&table[slot[i]], -1, e.id[i]);
        }
        again |= e.id[i] >= 0 && old[i] == e.id[i];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i * 32 < a.K && e.id[i] >= 0) table[slot[i]] = -1;
    e.repeated = __any_sync(0xffffffffu, again);
    if (e.repeated && a.tail) {  // a token has one probability: but for its first entry it is left out
        uint32_t out = 0;
        for (int k = 0; k < a.K; ++k) {
            int o = -1;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int of = __shfl_sync(0xffffffffu, e.id[i], k & 31);
                if (i == k >> 5) o = of;
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (k < i * 32 + lane && o == e.id[i] && o >= 0) out |= 1u << i;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (out >> i & 1) e.id[i] = -1;
        bad = true;
    }
    if (bad) report(a.status, ESTP_ERR_INVALID_ARG);
    const char* row = a.base + r * a.ld_bytes;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        e.z[i] = kBf16 ? 0xFF80u : 0xFF800000u;
        if (i * 32 < a.K && e.id[i] >= 0 && in_bounds(r < a.n_rows && e.id[i] < a.V, a.status))
            e.z[i] = kBf16 ? (uint32_t)reinterpret_cast<const uint16_t*>(row)[e.id[i]] : reinterpret_cast<const uint32_t*>(row)[e.id[i]];
        if (e.id[i] < 0) e.x[i] = -INFINITY;
    }
    __syncwarp();
}

template <bool kBf16>
__device__ __forceinline__ void put_entries(const DistillArgs& a, const Entries& e, Teacher& t) {
    const int lane = threadIdx.x & 31;
    float z[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) z[i] = __uint_as_float(kBf16 ? e.z[i] << 16 : e.z[i]);
    bool some = false;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        some |= e.id[i] >= 0;
        top = fmaxf(top, e.x[i]);
    }
    some = __any_sync(0xffffffffu, some);
    float q[kPer], lq[kPer];
    Two Q{0.f, 0.f}, rest{0.f, 0.f};
    if (a.tail) {
        // the q are rounded exponentials, but their sum and 1 less it add no error
        RowStat in = no_stat();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            lq[i] = e.x[i];
            q[i] = 0.f;
            if (i * 32 < a.K) {
                q[i] = expf(e.x[i]);
                Q = plus(Q, Two{q[i], 0.f});
                const bool bad = isnan(z[i]) || z[i] == INFINITY;
                if (e.id[i] >= 0) join(in, RowStat{z[i], bad ? NAN : z[i] == -INFINITY ? 0.f : 1.f, 0.f}, a.c);
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1)
            Q = plus(Q, Two{__shfl_xor_sync(0xffffffffu, Q.hi, off), __shfl_xor_sync(0xffffffffu, Q.lo, off)});
        Q = two_sum(Q.hi, Q.lo);
        if (some) {
            rest = two_sum(1.f, -Q.hi);
            rest = two_sum(rest.hi, rest.lo - Q.lo);
            if (rest.hi < 0.f) rest = Two{0.f, 0.f};
        }
        join_lanes<false>(in, a.c);
        t.in = in;
    } else {
        top = pivot(warp_max(top));
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            lq[i] = q[i] = 0.f;
            if (i * 32 < a.K) {
                lq[i] = (e.x[i] - top) / a.T;
                q[i] = expf(lq[i]);
                sum += q[i];
            }
        }
        sum = warp_sum(sum);
        const bool none = sum == 0.f;  // no entry, or only such of -inf
        const float l = none ? 0.f : logf(sum);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (i * 32 < a.K) {
                q[i] = none ? 0.f : q[i] / sum;
                lq[i] -= l;
            }
        Q.hi = none ? 0.f : 1.f;
        some = !none;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (i * 32 >= a.K) continue;
        const int j = i * 32 + lane;
        t.id[j] = e.id[i];
        t.q[j] = q[i];
        t.lq[j] = lq[i];
        t.z[j] = z[i];
    }
    if (lane == 0) {
        t.Q = Q.hi;
        t.rest = rest.hi;
        t.Q_lo = Q.lo;
        t.rest_lo = rest.lo;
        t.some = some;
        t.repeated = e.repeated;
        t.g = e.w / a.T;
    }
    __syncwarp();
}

// From the statistics `st` of every token, or with the tail of those that are not named.
__device__ __forceinline__ Factors row_factors(const DistillArgs& a, const Teacher& t, const RowStat& st) {
    Factors f;
    RowStat all = st;
    if (a.tail) join(all, t.in, a.c);
    f.m = pivot(all.m);
    f.s = all.s;
    f.empty = all.s == 0.f;
    f.zero = !t.some || t.g == 0.f;
    f.pivot = f.m;
    f.A = f.empty ? 0.f : t.g * t.Q / all.s;
    f.rest = t.rest;
    if (a.tail) {
        // Where the student has no other token, what the teacher leaves to them may be the rounding of its log
        // probabilities: sum q_j |x_j| 2^-24 + 2^-23 at most, below 2^-20 for the entropies that 128 tokens have.
        const bool no_other = st.s == 0.f;
        if (no_other && f.rest <= 0x1p-20f) f.rest = 0.f;
        // the exponentials of these elements are taken against the maximum that their own sum belongs to
        f.pivot = pivot(st.m);
        // (Q + q_r) / s - q_r / s_other over one denominator, where s = s_other + s_named: the terms that cancel are gone
        const float other = st.s * ex2(max_nan((f.pivot - f.m) * a.c, kCut));
        const float named = t.in.s * ex2(max_nan((t.in.m - f.m) * a.c, kCut));
        f.A = no_other || f.empty ? 0.f : t.g * ((t.Q * other - f.rest * named) / (all.s * st.s));
    }
    f.M = f.pivot * a.c;
    f.framed = near_frame(f.M);
    f.near = f.A * ex2(-frame_off(f.pivot, a.c));
    return f;
}

// ln x for x > 0 to about 1e-9: x = 2^k m with m in [3/4, 3/2), ln m = 2 artanh s with s = (m - 1) / (m + 1), |s| <= 1/5.
// s is carried in two floats, and so are k ln 2 (its first 12 bits times k are exact) and the sum; the series
// behind 2 s is below 0.006 and needs one.
__device__ __forceinline__ Two two_log(Two x) {
    const int b = __float_as_int(x.hi), k = (b - 0x3F400000) >> 23;
    const float m = __int_as_float(b - (k << 23)), ml = x.lo * __int_as_float((127 - k) << 23);
    const float n = m - 1.f;  // exact
    Two d = two_sum(m, 1.f);
    d.lo += ml;
    const float s = n / d.hi, sl = (__fmaf_rn(-s, d.hi, n) + (ml - s * d.lo)) / d.hi, w = s * s;
    float p = 1.f / 13.f;
    p = fmaf(p, w, 1.f / 11.f);
    p = fmaf(p, w, 1.f / 9.f);
    p = fmaf(p, w, 1.f / 7.f);
    p = fmaf(p, w, 1.f / 5.f);
    p = fmaf(p, w, 1.f / 3.f);
    constexpr float kHi = 2839.f / 4096.f, kLo = (float)(0.69314718055994531 - 2839. / 4096.);
    return plus(Two{(float)k * kHi, (float)k * kLo}, Two{2.f * s, 2.f * (sl + s * w * p)});
}

// One warp.  From the fp32 sums on in two floats: where student and teacher agree, or both leave nearly everything to the
// other tokens (a high temperature), the loss is a small difference of terms whose logarithms are off by 1e-6 in one
// float, and with them a loss of 1e-3 has three digits left.  (64-bit arithmetic does as well, but there are 2 such
// operations a clock on an SM: 2048 rows of 128256 took 210 us with it and 183 in two floats, one step apart.)
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Teacher& t, const RowStat& st, const Factors& f) {
    const int lane = threadIdx.x & 31;
    if (!t.some) return 0.f;
    Two sum{0.f, 0.f};
    float plain = 0.f;
    bool any = f.rest != 0.f;
    for (int j = lane; j < a.K; j += 32) {
        const float q = t.q[j], z = t.z[j];
        if (t.id[j] >= 0 && q != 0.f) {
            any = true;
            // (halves: the distance of two finite logits may overflow)
            const float term = q * t.lq[j] + q * (0.5f * f.m - 0.5f * z) / a.T * 2.f;
            plain += term;
            // q may be next to nothing where (z - m) / T is beyond a float's end, or so near it that a product of two
            // floats is infinity and its error -infinity: such a term in one float
            const Two y = times(two_sum(z, -f.m), a.inv_T);
            sum = plus(sum, fabsf(y.hi) < 1e30f ? times(Two{q, 0.f}, plus(Two{t.lq[j], 0.f}, Two{-y.hi, -y.lo})) : Two{term, 0.f});
        }
    }
    any = __any_sync(0xffffffffu, any);
    plain = warp_sum(plain);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        sum = plus(sum, Two{__shfl_xor_sync(0xffffffffu, sum.hi, off), __shfl_xor_sync(0xffffffffu, sum.lo, off)});
    if (f.empty) return any ? INFINITY : 0.f;
    if (f.rest != 0.f && st.s == 0.f) return INFINITY;
    // infinite, NaN, or near a float's end (tokens at the type's lowest value): in one float
    if (!(fabsf(plain) < 1e4f) || isnan(f.s) || (f.rest != 0.f && !(f.pivot - f.m > -1e30f))) {
        plain += t.Q * logf(f.s);
        if (f.rest != 0.f)
            plain += f.rest * (logf(f.rest) - logf(st.s) + logf(f.s)) + f.rest * (0.5f * f.m - 0.5f * f.pivot) / a.T * 2.f;
        return plain;
    }
    // ln of the sum, of what the teacher leaves to the others, and of what the student does: 1 - sum p_id while that is at
    // least a half, else by their own sum
    Two left{1.f, 0.f};
    bool direct = false;
    if (a.tail) {
        const float num = t.in.s * ex2(max_nan((t.in.m - f.m) * a.c, kCut)), named = num / f.s;
        direct = !(named <= 0.5f);
        left = two_sum(1.f, -named);
        left.lo -= __fmaf_rn(-named, f.s, num) / f.s;
        if (direct) left = Two{st.s, 0.f};
    }
    const Two rest{t.rest, t.rest_lo};
    const Two l = two_log(lane == 0 ? Two{f.s, 0.f} : lane == 1 ? rest : left);
    const Two ls{__shfl_sync(0xffffffffu, l.hi, 0), __shfl_sync(0xffffffffu, l.lo, 0)};
    sum = plus(sum, times(Two{t.Q, t.Q_lo}, ls));
    if (f.rest != 0.f) {
        const Two lrest{__shfl_sync(0xffffffffu, l.hi, 1), __shfl_sync(0xffffffffu, l.lo, 1)};
        Two lp{__shfl_sync(0xffffffffu, l.hi, 2), __shfl_sync(0xffffffffu, l.lo, 2)};
        if (direct) {
            lp = plus(plus(times(two_sum(f.pivot, -f.m), a.inv_T), lp), Two{-ls.hi, -ls.lo});
        }
        sum = plus(sum, times(rest, plus(lrest, Two{-lp.hi, -lp.lo})));
    }
    return sum.hi + sum.lo;
}

// The gradient at a named token, given what it would be were it not one.
__device__ __forceinline__ float named_grad(const DistillArgs& a, const Teacher& t, const Factors& f, int j, float x) {
    if (f.empty) return 0.f;
    if (!a.tail) return x - t.g * t.q[j];
    const float p = ex2(max_nan((t.z[j] - f.m) * a.c, kCut)) / f.s;
    return t.g * ((t.Q + f.rest) * p - t.q[j]);
}

// Calls f(j) in every lane for each token j of a unit.
template <class F>
__device__ __forceinline__ void each_named(const int32_t* ids, int K, int per, int unit, F f) {
    const int lane = threadIdx.x & 31;
    for (int i0 = 0; i0 < K; i0 += 32) {
        const int i = i0 + lane;
        const int id = i < K ? ids[i] : -1;
        uint32_t hit = __ballot_sync(0xffffffffu, id >= 0 && id / per == unit);
        while (hit) {
            const int j = i0 + __ffs(hit) - 1;
            hit &= hit - 1;
            f(j);
        }
    }
}

// Named tokens among a warp's 32 units from `unit` on become -inf; `lanes` marks the units.  (A call, so that the loops
// around it stay short: a row has K such units among thousands.)
template <bool kBf16>
__device__ __noinline__ uint4 mask_ids(const int32_t* ids, int K, uint32_t lanes, int unit, uint4 v) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31;
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
    while (lanes) {
        const int l = __ffs(lanes) - 1;
        lanes &= lanes - 1;
        each_named(ids, K, per, unit + l, [&](int j) {
            const int at = ids[j] - (unit + l) * per;
#pragma unroll
            for (int e = 0; e < per; ++e)
                if (lane == l && e == at) {
                    if (!kBf16) w[e] = 0xFF800000u;
                    else if (e & 1) w[e >> 1] = (w[e >> 1] & 0x0000FFFFu) | 0xFF800000u;
                    else w[e >> 1] = (w[e >> 1] & 0xFFFF0000u) | 0x0000FF80u;
                }
        });
    }
    return v;
}

template <bool kBf16, bool kFramed>
__device__ __forceinline__ void other_grad(const Factors& f, const uint4& v, float c, float (&x)[8]) {
    const float2 c2 = make_float2(c, c);
    const float2 off = kFramed ? make_float2(-f.M, -f.M) : make_float2(-f.pivot, -f.pivot);
    const float2 A2 = kFramed ? make_float2(f.near, f.near) : make_float2(f.A, f.A);
#pragma unroll
    for (int i = 0; i < (kBf16 ? 4 : 2); ++i) {
        const float2 d = kFramed ? __ffma2_rn(pair<kBf16>(v, i), c2, off) : __fmul2_rn(__fadd2_rn(pair<kBf16>(v, i), off), c2);
        const float2 g = __fmul2_rn(A2, make_float2(ex2(d.x), ex2(d.y)));
        x[2 * i] = g.x;
        x[2 * i + 1] = g.y;
    }
}

// ------------------------------------------------------------------ rows kept by a cluster
// A cluster of C CTAs takes a row, each a slice; up to three CTAs an SM, of different clusters, so that one
// computes while another waits.  Eight warps work on the slice: a thread copies its own units into
// shared memory (cp.async), reads them there for the statistics, and again for the gradient, after which it
// copies the next row's into their place: the next row is on its way while this one is written, and no
// barrier stands between a copy and its use.
//
// The ninth warp has the teacher's side of the next row ready, forms the loss, and one row later writes the named
// tokens' gradients over what the workers wrote there.
//
// One cluster barrier a row: before it each worker warp stores its statistics into every CTA of the cluster, after
// it every warp joins them for itself.
//
// One CTA an SM with the slices of two or three rows, the statistics a row ahead of the gradient and warps of their own for the
// joins and the teacher hides the barrier, but its 16 or 24 workers then do the same thing at the same time: 2048
// rows of 128256 tokens in 234 us and 1021 of 152064 with the tail in 185.
constexpr int kWork = 256;
constexpr int kWorkWarps = kWork / 32;
constexpr int kRowThreads = kWork + 32;
constexpr int kRowBlocks = 3;  // CTAs an SM at most
constexpr int kGroup = 3;      // units a worker has in registers at once (8: 215 us, the loops outgrow the instruction cache)
constexpr int kTeachers = 3;   // rows i - 1 .. i + 1
constexpr int kMaxCluster = 8;
constexpr int kSliceBytes = 200 * 1024;  // dynamic shared memory at most

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void store_remote(const void* p, uint32_t rank, float x, float y) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, %1;\n\t"
        "st.shared::cluster.v2.f32 [a], {%2, %3};\n\t}" ::"r"((uint32_t)__cvta_generic_to_shared(p)),
        "r"(rank), "f"(x), "f"(y)
        : "memory");
}

__device__ __forceinline__ void copy_unit(uint4* to, const char* from) {
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the thread's last `left` groups of copies are there.
__device__ __forceinline__ void copies_wait(int left) {
    switch (left) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}

// Elements of a unit whose bits are set in `marks` become -inf.
template <bool kBf16>
__device__ __forceinline__ uint4 mask_marked(uint4 v, uint32_t marks) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int e = 0; e < (kBf16 ? 8 : 4); ++e)
        if (marks >> e & 1) {
            if (!kBf16) w[e] = 0xFF800000u;
            else if (e & 1) w[e >> 1] = (w[e >> 1] & 0x0000FFFFu) | 0xFF800000u;
            else w[e >> 1] = (w[e >> 1] & 0xFFFF0000u) | 0x0000FF80u;
        }
    return v;
}

// The three forms of the kernel: the code of a row's loops should be short, as 27 warps in three places of it share an SM's
// instruction caches.  (One kernel for all: 2048 rows of 128256 tokens 183 us, by forms 179; 8192 of 32000 202 and 183.)
// With the tail, named tokens are not in the sums.  Making marks for them takes the ninth warp longer than it takes
// the workers to look a few tokens through: by tokens and by marks, us, 1021 rows of 152064 with 32 named 130 and
// 134, 2048 of 128256 with 64 209 and 208, 8192 of 32000 with 64 263 and 236.
constexpr int kTailFew = 1, kTailMarks = 2;
constexpr int kFewNamed = 32;

// Named tokens of a warp's 32 units become -inf: `units` marks the units that hold some, whose bytes of marks, a bit each,
// stand in their order from `first` on.
template <bool kBf16>
__device__ __noinline__ uint4 mask_named(uint4 v, uint32_t units, const uint8_t* first) {
    const int lane = threadIdx.x & 31;
    if (units >> lane & 1) v = mask_marked<kBf16>(v, first[__popc(units & ((1u << lane) - 1))]);
    return v;
}

// A CTA's slice of a row: n units, the row's u0-th on; a worker's are tid, tid + kWork, .. in groups of kGroup, the last
// one of what is left.
struct Slice {
    uint4* kept;
    const uint32_t* bits;   // with the tail: units that hold a named token, and behind them the place of each 32's first one
    int words;              // among
    const uint8_t* marks;
    int n, u0;
};

// Calls f(at, N) for each of the groups; every worker has all of a group's units, and all of them are whole, but for
// the last unit of the last group.
template <class F, int N = kGroup>
__device__ __forceinline__ void last_group(int left, int at, F& f) {
    if constexpr (N > 1) {
        if (left < N) {
            last_group<F, N - 1>(left, at, f);
            return;
        }
    }
    f(at, std::integral_constant<int, N>(), true);
}
template <class F>
__device__ __forceinline__ void each_group(int n, F f) {
    const int units = (n + kWork - 1) / kWork;  // of a worker, the last one not of all
    int u = 0;
    for (; u + kGroup < units; u += kGroup) f(u * kWork, std::integral_constant<int, kGroup>(), false);
    if (u < units) last_group(units - u, u * kWork, f);
}
__device__ __forceinline__ int groups_of(int n) { return ((n + kWork - 1) / kWork + kGroup - 1) / kGroup; }

// Copies N of the worker's units of row r, whose slice is at `from`.
template <int N>
__device__ __forceinline__ void copy_group(const DistillArgs& a, int64_t r, const Slice& s, int at, bool last, const char* from) {
    const int c = at + (int)threadIdx.x;
    const char* q = from + (int64_t)c * 16;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < N - 1 || !last || c + k * kWork < s.n) {
            const int u = c + k * kWork;
            if (units_there(a, r, s.u0 + u, s.u0 + u + 1, 1, false) && in_bounds(u < s.n, a.status))
                copy_unit(&s.kept[u], q + k * (kWork * 16));
        }
    copies_commit();
}

// N of the worker's units, from `at` on, into the statistics.
template <bool kBf16, int kTail, int N>
__device__ __forceinline__ void hold_units(const DistillArgs& a, const Teacher& t, const Slice& s, int at, bool last,
                                           LaneStat<false>& st) {
    constexpr int per = kBf16 ? 8 : 4;
    const int c = at + (int)threadIdx.x;
    uint4 v[N];
#pragma unroll
    for (int k = 0; k < N - 1; ++k) v[k] = s.kept[c + k * kWork];
    if (last) {
        const int l = c + (N - 1) * kWork, valid = a.V - (s.u0 + l) * per;
        v[N - 1] = l < s.n ? s.kept[l] : masked_unit<kBf16>();
        if (valid < per) mask_unit<kBf16>(v[N - 1], valid);
    } else {
        v[N - 1] = s.kept[c + (N - 1) * kWork];
    }
    if constexpr (kTail != 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int w = (c & ~31) + k * kWork;  // the warp's units
            const uint32_t units = w < s.n ? s.bits[w >> 5] : 0;
            if (units)
                v[k] = kTail == kTailMarks ? mask_named<kBf16>(v[k], units, s.marks + s.bits[s.words + (w >> 5)])
                                           : mask_ids<kBf16>(t.id, a.K, units, s.u0 + w, v[k]);
        }
    }
    st.template add_units<kBf16>(v, units_max<kBf16, N>(v), a.c);
}

// The gradient of N of them, of row r, and copies of row r + step (`next`, if any) into their place.
template <bool kBf16, bool kFramed, int N>
__device__ __forceinline__ void kept_grad(const DistillArgs& a, int64_t r, int64_t step, const Factors& f, const Slice& s, int at,
                                          bool last, char* out, const char* next) {
    constexpr int per = kBf16 ? 8 : 4;
    const int c = at + (int)threadIdx.x;
    char* p = out + (int64_t)c * 16;
    uint4 v[N];
#pragma unroll
    for (int k = 0; k < N - 1; ++k) v[k] = s.kept[c + k * kWork];
    v[N - 1] = last && c + (N - 1) * kWork >= s.n ? masked_unit<kBf16>() : s.kept[c + (N - 1) * kWork];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float x[8];
        other_grad<kBf16, kFramed>(f, v[k], a.c, x);
        const int u = c + k * kWork;
        if (k < N - 1 || !last) {
            if (units_there(a, r, s.u0 + u, s.u0 + u + 1, per, true) && in_bounds(u < s.n, a.status))
                store_whole<kBf16>(p + k * (kWork * 16), x);
        } else if (u < s.n && units_there(a, r, s.u0 + u, s.u0 + u + 1, per, false)) {
            store_unit<kBf16>(out, u, a.V - s.u0 * per, x);
        }
    }
    if (next) copy_group<N>(a, r + step, s, at, last, next);  // (every value has been used)
}

// The named tokens of a slice, over what an unnamed one would have there (a warp).
template <bool kBf16>
__device__ __forceinline__ void put_named(const DistillArgs& a, int64_t r, const Teacher& t, const Factors& f, int u0, int n) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31;
    if (f.zero) return;
    char* out = a.out + r * a.out_bytes;
    for (int j0 = 0; j0 < a.K; j0 += 32) {
        const int j = j0 + lane, id = j < a.K ? t.id[j] : -1;
        const unsigned u = (unsigned)(id / per - u0);
        const bool mine = id >= 0 && u < (unsigned)n;
        bool first = mine;
        float x = 0.f;
        if (mine && !a.tail) x = f.A * ex2(max_nan((t.z[j] - f.pivot) * a.c, kCut));
        if (!t.repeated || a.tail) {
            if (mine) x = named_grad(a, t, f, j, x);
        } else {  // a repeated token counts each time: its first place has the sum
            for (int k = 0; k < a.K; ++k)
                if (mine && t.id[k] == id) {
                    x = named_grad(a, t, f, k, x);
                    first &= k >= j;
                }
        }
        if (first && in_bounds(id < a.V && r < a.n_rows, a.status)) {
            if (kBf16) reinterpret_cast<__nv_bfloat16*>(out)[id] = __float2bfloat16_rn(x);
            else reinterpret_cast<float*>(out)[id] = x;
        }
    }
}

template <bool kBf16, int kTail>
__global__ void __launch_bounds__(kRowThreads, kRowBlocks) distill_rows_kernel(const DistillArgs args, int slice, int C) {
    constexpr int per = kBf16 ? 8 : 4;
    DistillArgs a = args;
    a.tail = kTail != 0;  // (known to the compiler)
    extern __shared__ uint4 room[];                 // [slice], then with the tail [2][2][words]
    __shared__ Teacher teachers[kTeachers];
    __shared__ float2 stats[2][kMaxCluster * kWorkWarps];  // m, s of each worker warp of the cluster, of two rows
    __shared__ int32_t table[kSlots];
    __shared__ Asked asked;
    __shared__ uint32_t marks[2][kK / 4], places;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x % C, words = (slice + 31) / 32;
    const int u0 = min(rank * slice, a.nvec), n = min(slice, a.nvec - u0);
    const int64_t r0 = blockIdx.x / C, step = gridDim.x / C;
    const int rows = r0 < a.n_rows ? (int)((a.n_rows - r0 + step - 1) / step) : 0;  // of this cluster
    uint32_t* bits = reinterpret_cast<uint32_t*>(room + slice);
    const bool works = warp < kWorkWarps;
    auto from = [&](int i) { return a.base + (r0 + i * step) * a.ld_bytes + (int64_t)u0 * 16; };
    auto next_of = [](int k) { return k + 1 == kTeachers ? 0 : k + 1; };

    Entries e;  // (ninth warp) of the next row to be put, with its logits; `asked` is of the one after it
    auto put = [&](int i, int at) {
        if (i >= rows) return;
        put_entries<kBf16>(a, e, teachers[at]);
    };
    auto fetch = [&](int i) {  // row i's entries, row i + 1's asked for
        if (i >= rows) return;
        take_entries(a, asked, e);
        if (i + 1 < rows) ask_entries(a, r0 + (i + 1) * step, asked);
        check_entries<kBf16>(a, r0 + i * step, e, table);
        // (the workers have looked at row i - 2, whose place this is)
        if (a.tail) {
            uint32_t *b = bits + (i & 1) * 2 * words, *place = b + words;
            for (int k = lane; k < words; k += 32) b[k] = 0;
            marks[i & 1][lane] = 0;
            if (lane == 0) places = 0;
            __syncwarp();
            unsigned u[kPer];
            uint32_t old[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                u[k] = (unsigned)(e.id[k] / per - u0);
                if (k * 32 >= a.K || e.id[k] < 0 || u[k] >= (unsigned)n) u[k] = ~0u;
                old[k] = u[k] != ~0u ? atomicOr(&b[u[k] >> 5], 1u << (u[k] & 31)) : 1u;
            }
            if (kTail != kTailMarks) return;
            __syncwarp();
#pragma unroll
            for (int k = 0; k < kPer; ++k)  // who was the first of 32 units gives them their places
                if (old[k] == 0) place[u[k] >> 5] = atomicAdd(&places, __popc(b[u[k] >> 5]));
            __syncwarp();
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (u[k] != ~0u) {
                    const uint32_t m = place[u[k] >> 5] + __popc(b[u[k] >> 5] & ((1u << (u[k] & 31)) - 1));
                    atomicOr(&marks[i & 1][m >> 2], 1u << ((m & 3) * 8 + e.id[k] % per));
                }
        }
    };
    const int groups = groups_of(n);
    if (works) {
        const Slice s{room, nullptr, 0, nullptr, n, u0};
        if (rows > 0) each_group(n, [&](int at, auto N, bool last) { copy_group<decltype(N)::value>(a, r0, s, at, last, from(0)); });
    } else {
        for (int i = lane; i < kSlots; i += 32) table[i] = -1;
        __syncwarp();
        if (rows > 0) ask_entries(a, r0, asked);
        fetch(0);
        put(0, 0);
        fetch(1);
    }
    __syncwarp();
    cluster_sync();  // every CTA of the cluster runs before another one stores into its shared memory
    Factors f{};
    int before = 0;
    for (int i = 0, k = 0; i < rows; ++i, k = next_of(k)) {
        const Teacher& t = teachers[k];
        const Slice s{room, bits + (i & 1) * 2 * words, words, reinterpret_cast<const uint8_t*>(marks[i & 1]), n, u0};
        float2* mine = stats[i & 1];
        if (works) {
            LaneStat<false> st;
            int left = groups;
            each_group(n, [&](int at, auto N, bool last) {
                copies_wait(--left);
                hold_units<kBf16, kTail, decltype(N)::value>(a, t, s, at, last, st);
            });
            RowStat x = st.row(a.c);
            join_lanes<false>(x, a.c);
            if (lane < C && in_bounds(C <= kMaxCluster && rank * kWorkWarps + warp < C * kWorkWarps, a.status))
                store_remote(&mine[rank * kWorkWarps + warp], lane, x.m, x.s);
        } else {
            put(i + 1, next_of(k));
        }
        __syncwarp();
        cluster_sync();
        RowStat st = no_stat();
        for (int w = lane; w < C * kWorkWarps; w += 32) {
            if (w < 32) st = RowStat{mine[w].x, mine[w].y, 0.f};
            else join(st, RowStat{mine[w].x, mine[w].y, 0.f}, a.c);
        }
        __syncwarp();
        join_lanes<false>(st, a.c);
        if (!works) {
            // (the workers' gradient of the row before is behind the barrier)
            if (i > 0) put_named<kBf16>(a, r0 + (i - 1) * step, teachers[before], f, u0, n);
            f = row_factors(a, t, st);
            if (rank == 0) put_loss(a, r0 + i * step, row_loss(a, t, st, f));
            before = k;
            fetch(i + 2);
        } else {
            f = row_factors(a, t, st);
            const int64_t r = r0 + i * step;
            char* out = a.out + r * a.out_bytes + (int64_t)u0 * 16;
            const char* next = i + 1 < rows ? from(i + 1) : nullptr;
            if (f.zero) {
                const float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (int c = tid; c < n; c += kWork)
                    if (units_there(a, r, u0 + c, u0 + c + 1, per, false)) store_unit<kBf16>(out, c, a.V - u0 * per, x);
                if (next) each_group(n, [&](int at, auto N, bool last) { copy_group<decltype(N)::value>(a, r + step, s, at, last, next); });
            } else if (f.framed) {
                each_group(n, [&](int at, auto N, bool last) { kept_grad<kBf16, true, decltype(N)::value>(a, r, step, f, s, at, last, out, next); });
            } else {
                each_group(n, [&](int at, auto N, bool last) { kept_grad<kBf16, false, decltype(N)::value>(a, r, step, f, s, at, last, out, next); });
            }
        }
        __syncwarp();
    }
    __syncthreads();  // the last row's stores
    if (!works && rows > 0) put_named<kBf16>(a, r0 + (rows - 1) * step, teachers[before], f, u0, n);
}

// ------------------------------------------------------------------ the loss alone
// A warp an equal piece of the flat run of units (vocab.cuh); of a row cut between warps each leaves its
// statistics, and the one that leaves the last joins them in order and forms the loss.  1024 rows of 152064 tokens with 100
// teacher logits in 63 to 66 us, 46 of bytes (clusters as above: 75 to 105).
struct EvalArgs {
    DistillArgs d;
    VocabRows rows;
    float4* part;      // [pieces][2]: m, s of a piece's first and last row
    uint32_t* count;   // by a row's first piece; zero between launches
};

// A byte for each unit of a chunk, a bit for each named token in it (a warp's own).
constexpr int kChunkUnits = 1024;
struct Marks {
    uint4 of[kChunkUnits / 16];
};

// Units [c0, c1) of a row; with the tail, named tokens do not count.  (Looking each marked unit up among the K tokens instead
// took 8192 rows of 32000 tokens with 64 named from 125 us to 176.)
template <bool kBf16>
__device__ __forceinline__ RowStat eval_units(const DistillArgs& a, const char* row, int c0, int c1, const int32_t* ids,
                                              Marks& marks) {
    constexpr int per = kBf16 ? 8 : 4;
    const int lane = threadIdx.x & 31, whole = min(c1, a.V / per);
    LaneStat<false> st;
    for (int chunk = c0; chunk < c1; chunk += kChunkUnits) {
        const int stop = min(c1, chunk + kChunkUnits);
        uint32_t steps = 0;  // the chunk's 32s of units that hold one
        if (a.tail) {
            __syncwarp();
            marks.of[lane] = marks.of[32 + lane] = make_uint4(0, 0, 0, 0);
            __syncwarp();
            for (int j = lane; j < a.K; j += 32) {
                const int id = ids[j];
                const unsigned k = (unsigned)(id / per - chunk);
                if (id >= 0 && k < (unsigned)kChunkUnits)
                    atomicOr(reinterpret_cast<uint32_t*>(marks.of) + (k >> 2), 1u << ((k & 3) * 8 + id % per));
            }
            __syncwarp();
            const uint4 x = marks.of[2 * lane], y = marks.of[2 * lane + 1];
            steps = __ballot_sync(0xffffffffu, (x.x | x.y | x.z | x.w | y.x | y.y | y.z | y.w) != 0);
        }
        for (int b = chunk; b < stop; b += 32 * kVocabUnroll) {
            uint4 v[kVocabUnroll];
            if (b + 32 * kVocabUnroll <= whole) {
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) v[k] = ld_once(row + (int64_t)(b + 32 * k + lane) * 16);
            } else {
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) v[k] = load_unit<kBf16>(row, b + 32 * k + lane, stop, a.V);
            }
            const uint32_t some = steps >> ((b - chunk) / 32);
            if (some & ((1u << kVocabUnroll) - 1)) {
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k)
                    if (some >> k & 1)
                        v[k] = mask_marked<kBf16>(v[k], reinterpret_cast<const uint8_t*>(marks.of)[b - chunk + 32 * k + lane]);
            }
            st.template add_units<kBf16>(v, units_max<kBf16, kVocabUnroll>(v), a.c);
        }
    }
    RowStat x = st.row(a.c);
    join_lanes<false>(x, a.c);
    return x;
}

template <bool kBf16, bool kTail>
__global__ void __launch_bounds__(kVocabThreads, kVocabBlocks) distill_eval_kernel(const EvalArgs a) {
    constexpr int kWarps = kVocabThreads / 32;
    __shared__ Teacher teachers[kWarps];
    __shared__ Asked asked[kWarps];
    __shared__ int32_t tables[kWarps][kSlots];
    __shared__ Marks marks[kWarps];
    DistillArgs d = a.d;
    d.tail = kTail;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
    if (w >= a.rows.pieces) return;
    const int64_t start = piece_start(a.rows, w), end = piece_start(a.rows, w + 1);
    for (int i = lane; i < kSlots; i += 32) tables[warp][i] = -1;
    __syncwarp();
    for (int64_t u = start; u < end;) {
        const int64_t r = quotient(u, a.rows.nvec), u0 = r * a.rows.nvec;
        const int c0 = (int)(u - u0), c1 = (int)(min(end, u0 + a.rows.nvec) - u0);
        const char* row = d.base + r * d.ld_bytes;
        if (!units_there(d, r, c0, c1, 1, false)) return;
        Entries e;
        ask_entries(d, r, asked[warp]);
        if (d.tail) {
            copies_done();
            __syncwarp();
        }
        RowStat st = eval_units<kBf16>(d, row, c0, c1, asked[warp].id, marks[warp]);
        bool write = true;
        if (c0 != 0 || c1 != a.rows.nvec) {
            const int64_t slot = w * 2 + (u == start ? 0 : 1);
            const int64_t lo = piece_of(a.rows, u0), hi = piece_of(a.rows, u0 + a.rows.nvec - 1);
            const int n = (int)(hi - lo + 1);
            write = false;
            if (in_bounds(lo >= 0 && slot < 2 * a.rows.pieces, d.status)) {
                if (lane == 0) a.part[slot] = make_float4(st.m, st.s, 0.f, 0.f);
                write = arrive(a.count + lo, n);
            }
            if (write) {
                st = no_stat();
                for (int i = lane; i < n; i += 32) {
                    const int64_t at = i ? (lo + i) * 2 : lo * 2 + (piece_start(a.rows, lo) < u0 ? 1 : 0);
                    if (!in_bounds(at < 2 * a.rows.pieces, d.status)) break;
                    const float4 x = __ldcg(&a.part[at]);
                    join(st, RowStat{x.x, x.y, 0.f}, d.c);
                }
                __syncwarp();
                join_lanes<false>(st, d.c);
            }
        }
        if (write) {
            Teacher& t = teachers[warp];
            take_entries(d, asked[warp], e);
            check_entries<kBf16>(d, r, e, tables[warp]);
            put_entries<kBf16>(d, e, t);
            put_loss(d, r, row_loss(d, t, st, row_factors(d, t, st)));
        }
        copies_done();
        __syncwarp();
        u = u0 + c1;
    }
}

// ------------------------------------------------------------------ many short rows
// A warp a row: both passes read it from memory, the second from the caches.  Where a row is a few KB, a cluster's
// barriers and its ninth warp take longer than the row.  By clusters and so, us: 8192 bf16 rows of 1000 tokens 85 and
// 28, of 2500 88 and 41, 7880 of 4707 (589 units) 100 and 66, 8192 of 8000 105 and 105; 1000 of 4707 25 and 28.  (Calls back
// to back, without the host: 8192 of 1000 22, 30000 of 4000 190, for 5 and 72 of bytes: in a warp the teacher's side, the
// stream, the loss and the write stand one after another.)
constexpr int kShortUnits = 256;    // at most, with a row for every sixth warp
constexpr int kManyShortUnits = 640;  // at most, with one for every warp

template <bool kBf16, bool kFramed>
__device__ __forceinline__ void short_grad(const DistillArgs& a, int64_t r, const Factors& f, const char* row, char* out) {
    constexpr int N = 4;
    const int lane = threadIdx.x & 31;
    for (int b = lane; b < a.nvec; b += 32 * N) {
        uint4 v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = load_unit<kBf16>(row, b + 32 * k, a.nvec, a.V);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float x[8];
            other_grad<kBf16, kFramed>(f, v[k], a.c, x);
            if (b + 32 * k < a.nvec && units_there(a, r, b + 32 * k, b + 32 * k + 1, 1, false)) store_unit<kBf16>(out, b + 32 * k, a.V, x);
        }
    }
}

template <bool kBf16, bool kTail>
__global__ void __launch_bounds__(kVocabThreads, kVocabBlocks) distill_short_kernel(const DistillArgs args) {
    DistillArgs a = args;
    a.tail = kTail;
    constexpr int kWarps = kVocabThreads / 32;
    __shared__ Teacher teachers[kWarps];
    __shared__ Asked asked[kWarps];
    __shared__ int32_t tables[kWarps][kSlots];
    __shared__ Marks marks[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t step = (int64_t)gridDim.x * kWarps;
    int64_t r = (int64_t)blockIdx.x * kWarps + warp;
    Teacher& t = teachers[warp];
    for (int i = lane; i < kSlots; i += 32) tables[warp][i] = -1;
    __syncwarp();
    ask_entries(a, r, asked[warp]);
    for (; r < a.n_rows; r += step) {
        const char* row = a.base + r * a.ld_bytes;
        if (!units_there(a, r, 0, a.nvec, 1, false)) return;
        Entries e;
        take_entries(a, asked[warp], e);
        check_entries<kBf16>(a, r, e, tables[warp]);
        const RowStat st = eval_units<kBf16>(a, row, 0, a.nvec, asked[warp].id, marks[warp]);
        __syncwarp();
        ask_entries(a, r + step, asked[warp]);
        if (r + step < a.n_rows) fetch_units(row + step * a.ld_bytes, 0, a.nvec, a.nvec);
        put_entries<kBf16>(a, e, t);
        const Factors f = row_factors(a, t, st);
        put_loss(a, r, row_loss(a, t, st, f));
        char* out = a.out + r * a.out_bytes;
        if (f.zero) {
            const float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int c = lane; c < a.nvec; c += 32) store_unit<kBf16>(out, c, a.V, x);
        } else if (f.framed) {
            short_grad<kBf16, true>(a, r, f, row, out);
        } else {
            short_grad<kBf16, false>(a, r, f, row, out);
        }
        __syncwarp();  // the named tokens go over these
        put_named<kBf16>(a, r, t, f, 0, a.nvec);
        __syncwarp();
    }
}

// ------------------------------------------------------------------ longer rows
// A block takes a row in two passes; named units are marked for a span of it at a time.
constexpr int kLongThreads = 512;
constexpr int kLongWarps = kLongThreads / 32;
constexpr int kSpanUnits = 1 << 16;

template <bool kBf16>
__global__ void __launch_bounds__(kLongThreads) distill_long_kernel(const DistillArgs a) {
    constexpr int per = kBf16 ? 8 : 4, kStep = 32 * kVocabUnroll;
    __shared__ Teacher t;
    __shared__ uint32_t bits[kSpanUnits / 32];
    __shared__ RowStat part[kLongWarps];
    __shared__ int32_t table[kSlots];
    __shared__ Asked asked;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < kSpanUnits / 32; i += kLongThreads) bits[i] = 0;
    for (int i = tid; i < kSlots; i += kLongThreads) table[i] = -1;
    auto mark = [&](int span, bool set) {
        for (int j = tid; j < a.K; j += kLongThreads) {
            const unsigned k = (unsigned)(t.id[j] / per - span);
            if (t.id[j] >= 0 && k < (unsigned)kSpanUnits) {
                if (set) atomicOr(&bits[k >> 5], 1u << (k & 31));
                else bits[k >> 5] = 0;
            }
        }
        __syncthreads();
    };
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        const char* row = a.base + r * a.ld_bytes;
        __syncthreads();
        if (warp == 0) {
            Entries e;
            ask_entries(a, r, asked);
            take_entries(a, asked, e);
            check_entries<kBf16>(a, r, e, table);
            put_entries<kBf16>(a, e, t);
        }
        __syncthreads();
        LaneStat<false> st;
        for (int span = 0; span < a.nvec; span += kSpanUnits) {
            const int stop = min(a.nvec, span + kSpanUnits);
            mark(span, true);
            for (int b = span + warp * kStep; b < stop; b += kLongWarps * kStep) {
                uint4 v[kVocabUnroll];
                const bool there = units_there(a, r, b, stop, per, false);
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) v[k] = load_unit<kBf16>(row, b + 32 * k + lane, there ? stop : b, a.V);
                if (a.tail) {
#pragma unroll
                    for (int k = 0; k < kVocabUnroll; ++k) {
                        const int c = b + 32 * k;
                        const uint32_t lanes = c < stop ? bits[(c - span) >> 5] : 0;
                        if (lanes) v[k] = mask_ids<kBf16>(t.id, a.K, lanes, c, v[k]);
                    }
                }
                st.template add_units<kBf16>(v, units_max<kBf16, kVocabUnroll>(v), a.c);
            }
            __syncthreads();
            mark(span, false);
        }
        RowStat s = st.row(a.c);
        join_lanes(s, a.c);
        if (lane == 0) part[warp] = s;
        __syncthreads();
        RowStat all = lane < kLongWarps ? part[lane] : no_stat();
        join_lanes(all, a.c);
        const Factors f = row_factors(a, t, all);
        if (warp == 0) put_loss(a, r, row_loss(a, t, all, f));
        char* out = a.out + r * a.out_bytes;
        for (int span = 0; span < a.nvec; span += kSpanUnits) {
            const int stop = min(a.nvec, span + kSpanUnits);
            mark(span, true);
            for (int c = span + warp * 32; c < stop; c += kLongThreads) {
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (!f.zero) {
                    other_grad<kBf16, false>(f, load_unit<kBf16>(row, c + lane, stop, a.V), a.c, x);
                    const uint32_t lanes = bits[(c - span) >> 5];
                    for (uint32_t left = lanes; left; left &= left - 1) {
                        const int l = __ffs(left) - 1;
                        each_named(t.id, a.K, per, c + l, [&](int j) {
#pragma unroll
                            for (int e = 0; e < per; ++e)
                                if (lane == l && (c + l) * per + e == t.id[j]) x[e] = named_grad(a, t, f, j, x[e]);
                        });
                    }
                }
                if (c + lane < stop && units_there(a, r, c + lane, c + lane + 1, per, false)) store_unit<kBf16>(out, c + lane, a.V, x);
            }
            __syncthreads();
            mark(span, false);
        }
    }
}

// ------------------------------------------------------------------ launch
using RowsKernel = void (*)(DistillArgs, int, int);

size_t rows_bytes(int nvec, int C, bool tail) {
    const size_t slice = (size_t)((nvec + C - 1) / C);
    return slice * 16 + (tail ? 4 * ((slice + 31) / 32) * sizeof(uint32_t) : 0);
}

// Raises a kernel's shared memory limit and finds what CTAs that share an SM leave each other; once a context.
cudaError_t set_rows(estp_ctx* ctx, RowsKernel kernel, int which) {
    if (ctx->distill_set >> which & 1) return cudaSuccess;
    cudaFuncAttributes has;
    int sm = 0, system = 0;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSliceBytes);
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&has, kernel);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sm, cudaDevAttrMaxSharedMemoryPerMultiprocessor, ctx->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&system, cudaDevAttrReservedSharedMemoryPerBlock, ctx->device);
    if (e != cudaSuccess) return e;
    for (int n = 1; n <= kRowBlocks; ++n)
        ctx->distill_room[which][n - 1] = cta_room(sm, (int)has.sharedSizeBytes + system, n, kSliceBytes);
    ctx->distill_set |= 1u << which;
    return cudaSuccess;
}

// Launch of `clusters` clusters of C CTAs.
struct ClusterLaunch {
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = {};
    ClusterLaunch(int C, int clusters, size_t bytes, cudaStream_t st) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)C;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3((unsigned)(C * clusters));
        cfg.blockDim = dim3(kRowThreads);
        cfg.dynamicSmemBytes = bytes;
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
};

// Clusters of C that the GPU holds at once, asked once for each kernel, C and number of CTAs an SM: for the most shared
// memory of so many CTAs, so that the answer does not depend on the call that asked.
cudaError_t clusters_at_once(estp_ctx* ctx, RowsKernel kernel, int which, int C, int per_sm, int* fit) {
    int& known = ctx->distill_clusters[which][per_sm - 1][C - 1];
    if (known == 0) {
        ClusterLaunch l(C, ctx->num_sms, (size_t)ctx->distill_room[which][per_sm - 1], nullptr);
        int n = 0;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kernel, &l.cfg);
        if (e != cudaSuccess) return e;
        known = n > 0 ? n : -1;  // -1: no such cluster here
    }
    *fit = known;
    return cudaSuccess;
}

}  // namespace

estp_status launch_distill_loss(estp_ctx* ctx, const void* logits, estp_dtype dtype, int64_t n_rows, int64_t V,
                                int64_t ld, const int32_t* ids, const float* teacher, int K, float T, bool tail,
                                const float* weight, float* loss, void* out, int64_t ld_out, cudaStream_t st) {
    DistillArgs a;
    const bool bf16 = dtype == ESTP_BF16;
    const int per = 16 / esize(dtype);
    a.base = static_cast<const char*>(logits);
    a.ld_bytes = ld * esize(dtype);
    a.n_rows = n_rows;
    a.V = (int32_t)V;
    a.nvec = (int32_t)((V + per - 1) / per);
    a.ids = ids;
    a.teacher = teacher;
    a.K = K;
    a.tail = tail;
    a.T = T;
    a.c = (float)(1.4426950408889634 / (double)T);
    const double inv_T = 1. / (double)T;
    a.inv_T = Two{(float)inv_T, (float)(inv_T - (double)(float)inv_T)};
    a.weight = weight;
    a.loss = loss;
    a.out = static_cast<char*>(out);
    a.out_bytes = ld_out * esize(dtype);
    a.status = ctx->status;
    cudaError_t e;
    constexpr int kWarps = kVocabThreads / 32;

    if (!out) {
        EvalArgs v;
        v.d = a;
        v.rows = vocab_rows(ctx, logits, dtype, n_rows, V, ld, 32 * kVocabUnroll, kVocabBlocks);
        v.part = ctx->vocab_part;
        v.count = ctx->vocab_count;
        const unsigned blocks = (unsigned)((v.rows.pieces + kWarps - 1) / kWarps);
        if (bf16 && tail) distill_eval_kernel<true, true><<<blocks, kVocabThreads, 0, st>>>(v);
        else if (bf16) distill_eval_kernel<true, false><<<blocks, kVocabThreads, 0, st>>>(v);
        else if (tail) distill_eval_kernel<false, true><<<blocks, kVocabThreads, 0, st>>>(v);
        else distill_eval_kernel<false, false><<<blocks, kVocabThreads, 0, st>>>(v);
        e = cudaGetLastError();
        return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "distillation launch");
    }

    const int64_t at_once = (int64_t)ctx->num_sms * kVocabBlocks * kWarps;
    if (a.nvec <= kManyShortUnits && n_rows * 6 >= at_once && (a.nvec <= kShortUnits || n_rows >= at_once)) {
        const int64_t want = (n_rows + kWarps - 1) / kWarps, most = (int64_t)ctx->num_sms * kVocabBlocks;
        const unsigned blocks = (unsigned)(want < most ? want : most);
        if (bf16 && tail) distill_short_kernel<true, true><<<blocks, kVocabThreads, 0, st>>>(a);
        else if (bf16) distill_short_kernel<true, false><<<blocks, kVocabThreads, 0, st>>>(a);
        else if (tail) distill_short_kernel<false, true><<<blocks, kVocabThreads, 0, st>>>(a);
        else distill_short_kernel<false, false><<<blocks, kVocabThreads, 0, st>>>(a);
        e = cudaGetLastError();
        return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "distillation launch");
    }

    // The cluster size by what a wave of rows takes: a unit's share of an SM's part of the memory's rate (0.72 ns for
    // its read and its write) on the CTAs that share an SM, of which one by itself reaches some 0.4, and 2 us a row.
    const int kind = !tail ? 0 : K <= kFewNamed ? kTailFew : kTailMarks, which = 2 * kind + bf16;
    constexpr RowsKernel kernels[] = {distill_rows_kernel<false, 0>, distill_rows_kernel<true, 0>,
                                      distill_rows_kernel<false, kTailFew>, distill_rows_kernel<true, kTailFew>,
                                      distill_rows_kernel<false, kTailMarks>, distill_rows_kernel<true, kTailMarks>};
    const RowsKernel kernel = kernels[which];
    e = set_rows(ctx, kernel, which);
    if (e != cudaSuccess) return cuda_fail(e, "distillation kernel's shared memory");
    int C = 0, clusters = 0;
    double best = 0.;
    for (int c = 1; c <= kMaxCluster; ++c) {
        const int per_sm = ctas_of((int64_t)rows_bytes(a.nvec, c, tail), ctx->distill_room[which], kRowBlocks);
        if (per_sm < 1) continue;
        int fit = 0;
        e = clusters_at_once(ctx, kernel, which, c, per_sm, &fit);
        if (e != cudaSuccess) return cuda_fail(e, "distillation clusters");
        if (fit < 1) continue;
        const int64_t share = (n_rows * c + ctx->num_sms - 1) / ctx->num_sms;  // CTAs an SM really has
        const double together = share < per_sm ? (double)share : (double)per_sm;
        const double cost = (double)((n_rows + fit - 1) / fit) *
                            (0.72 * ((a.nvec + c - 1) / c) * (together < 2.5 ? 2.5 : together) + 2000.);
        if (C == 0 || cost < best) {
            best = cost;
            C = c;
            clusters = n_rows < fit ? (int)n_rows : fit;
        }
    }
    if (C == 0) {  // longer than the largest cluster keeps
        const int64_t most = (int64_t)ctx->num_sms * 2;
        const unsigned blocks = (unsigned)(n_rows < most ? n_rows : most);
        if (bf16) distill_long_kernel<true><<<blocks, kLongThreads, 0, st>>>(a);
        else distill_long_kernel<false><<<blocks, kLongThreads, 0, st>>>(a);
        e = cudaGetLastError();
    } else {
        ClusterLaunch l(C, clusters, rows_bytes(a.nvec, C, tail), st);
        e = cudaLaunchKernelEx(&l.cfg, kernel, a, (a.nvec + C - 1) / C, C);
    }
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "distillation launch");
}

}  // namespace estp
