// What the kernels over rows of logits share: the flat cut of the rows, the running softmax
// statistics of a warp, and the list of a row's greatest logits.
//
// For a row z of V logits and a temperature T, with m = max z and c = log2(e) / T,
//   d_v = (z_v - m) c,  s = sum 2^d_v,  t = sum 2^d_v d_v
// give ln p_v = (z_v - m) / T - ln s and the entropy ln s - ln2 t / s.  m is kept in the
// logits' own units: the difference z_v - m is then exact where it counts (z_v near m) and a row of
// the type's lowest values does not overflow before it is subtracted.  d is cut off at -200, where
// 2^d is 0: so a masked logit of -inf adds 0 to t instead of 0 * -inf.  NaN passes the cut-off
// (max.NaN), and +inf gives inf - inf, so that a row which holds either has a NaN sum.
#pragma once

#include "estp_internal.cuh"

namespace estp {

constexpr int kVocabThreads = 256;
constexpr int kVocabBlocks = 3;       // resident blocks an SM the registers of the streams are sized for: 80 a thread
constexpr int kVocabUnroll = 8;       // 16-byte loads a lane has in flight: 96 KB an SM, twice what its share of the memory's rate needs
constexpr int kMaxAlternatives = 128;  // entries of a row's list
constexpr int64_t kMaxVocab = 1 << 26;  // the index of a row's 16-byte unit in 24 bits
constexpr float kMinTemperature = 1e-6f;  // log2(e) / T stays far from overflow
constexpr float kCut = -200.f;

__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// ------------------------------------------------------------------ the flat cut
// The rows as one run of 16-byte units, cut into equal pieces, a warp each: every warp streams the
// same number of bytes whatever V and n_rows are.  (The first `more` pieces have a unit more.)  Or each row into
// `per_row` pieces.
struct VocabRows {
    const char* base;
    int64_t ld_bytes;
    int64_t n_rows;
    int64_t units;   // n_rows * nvec
    int64_t pieces;
    int64_t q, more;
    int32_t V;
    int32_t nvec;    // units of a row (the last one may be partial)
    int32_t per_row; // 0: equal pieces of all rows
};

// Quotients of what nearly always fits 32 bits: a 64-bit division takes some hundred instructions, and
// a warp makes several before its first load.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return (((uint64_t)a | (uint64_t)b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

__device__ __forceinline__ int64_t piece_start(const VocabRows& a, int64_t w) {
    if (a.per_row) {
        const uint32_t r = (uint32_t)w / (uint32_t)a.per_row, i = (uint32_t)w - r * (uint32_t)a.per_row;
        return (int64_t)r * a.nvec + (uint32_t)a.nvec * i / (uint32_t)a.per_row;  // (both below 2^16 and 2^24: see vocab_rows)
    }
    return w * a.q + (w < a.more ? w : a.more);
}

// The last piece that starts at or before unit u.
__device__ __forceinline__ int64_t piece_of(const VocabRows& a, int64_t u) {
    if (a.per_row) {
        const int64_t r = quotient(u, a.nvec);
        return r * a.per_row + ((uint32_t)(u - r * a.nvec + 1) * (uint32_t)a.per_row - 1) / (uint32_t)a.nvec;
    }
    const int64_t b = a.more * (a.q + 1);
    return u < b ? quotient(u, a.q + 1) : a.more + quotient(u - b, a.q);
}

inline void cut_rows(VocabRows& a, int64_t pieces, int per_row) {
    a.pieces = pieces;
    a.per_row = per_row;
    a.q = a.units / pieces;
    a.more = a.units % pieces;
}

inline VocabRows vocab_rows(const estp_ctx* ctx, const void* logits, estp_dtype dtype, int64_t n_rows, int64_t V,
                            int64_t ld, int min_units, int blocks) {
    VocabRows a;
    const int per = 16 / esize(dtype);
    a.base = static_cast<const char*>(logits);
    a.ld_bytes = ld * esize(dtype);
    a.n_rows = n_rows;
    a.V = (int32_t)V;
    a.nvec = (int32_t)((V + per - 1) / per);
    a.units = n_rows * a.nvec;
    const int64_t most = (int64_t)ctx->num_sms * blocks * (kVocabThreads / 32);
    const int64_t want = (a.units + min_units - 1) / min_units;
    cut_rows(a, want < most ? want : most, 0);
    return a;
}

// --------------------------------------------------------------- running statistics
struct RowStat {
    float m, s, t;
};

__device__ __forceinline__ RowStat no_stat() { return RowStat{-INFINITY, 0.f, 0.f}; }
__device__ __forceinline__ float pivot(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ void join(RowStat& a, const RowStat& b, float c) {
    const float m = fmaxf(a.m, b.m), p = pivot(m);
    const float da = max_nan((a.m - p) * c, kCut), db = max_nan((b.m - p) * c, kCut);
    const float fa = ex2(da), fb = ex2(db);
    a.t = fa * fmaf(da, a.s, a.t) + fb * fmaf(db, b.s, b.t);
    a.s = fa * a.s + fb * b.s;
    a.m = m;
}

// The lanes' statistics joined: the maximum first, then sums against it.
template <bool kT = true>
__device__ __forceinline__ void join_lanes(RowStat& a, float c) {
    float m = a.m;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    const float d = max_nan((a.m - pivot(m)) * c, kCut), f = ex2(d);
    float s = f * a.s, t = f * fmaf(d, a.s, a.t);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, off);
        if (kT) t += __shfl_xor_sync(0xffffffffu, t, off);
    }
    a = RowStat{m, s, t};
}

// Greatest logit of N units (NaN is passed over: the sums show it).
template <bool kBf16, int N>
__device__ __forceinline__ float units_max(const uint4* v) {
    if (kBf16) {
        __nv_bfloat162 x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v[k]);
            x[k] = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        }
#pragma unroll
        for (int w = 1; w < N; w *= 2)
#pragma unroll
            for (int k = 0; k + w < N; k += 2 * w) x[k] = __hmax2(x[k], x[k + w]);
        return fmaxf(__low2float(x[0]), __high2float(x[0]));
    }
    float x = -INFINITY;
#pragma unroll
    for (int k = 0; k < N; ++k)
        x = fmaxf(x, fmaxf(fmaxf(__uint_as_float(v[k].x), __uint_as_float(v[k].y)), fmaxf(__uint_as_float(v[k].z), __uint_as_float(v[k].w))));
    return x;
}

// The maxima of N units of a lane, of which bf16 ones stay a pair each.
template <bool kBf16, int N>
struct UnitMaxima {
    __nv_bfloat162 x[kBf16 ? N : 1];
    float y[kBf16 ? 1 : N];
    __device__ __forceinline__ explicit UnitMaxima(const uint4 (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v[k]);
            if constexpr (kBf16) x[k] = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
            else y[k] = units_max<false, 1>(&v[k]);
        }
    }
    __device__ __forceinline__ float all() const {
        if constexpr (kBf16) {
            __nv_bfloat162 m = x[0];
#pragma unroll
            for (int k = 1; k < N; ++k) m = __hmax2(m, x[k]);
            return fmaxf(__low2float(m), __high2float(m));
        } else {
            float m = y[0];
#pragma unroll
            for (int k = 1; k < N; ++k) m = fmaxf(m, y[k]);
            return m;
        }
    }
    // The units that hold a logit of at least `bound`, a bit each (a bf16 logit reaches what rounds up to it).
    __device__ __forceinline__ uint32_t reached(float bound) const {
        uint32_t hits = 0;
        const __nv_bfloat162 b = __bfloat162bfloat162(__float2bfloat16_ru(bound));
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if constexpr (kBf16) hits |= __hge2_mask(x[k], b) != 0u ? 1u << k : 0u;
            else hits |= y[k] >= bound ? 1u << k : 0u;
        }
        return hits;
    }
};

// Two consecutive elements of a unit, as fp32.
template <bool kBf16>
__device__ __forceinline__ float2 pair(const uint4& v, int i) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
    if (kBf16) return make_float2(bf16lo(w[i]), bf16hi(w[i]));
    return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}

// The near frame.  d = (z - m) c costs an addition and a product; z c - M with M = m c rounded is one
// fused operation, and off by the same delta = m c - M (which fma(m, c, -M) gives) in every term: 2^d
// by the factor 2^delta.  Where |M| <= 2^20 delta is at most 1/16, and sums in that frame
// are brought back exactly enough: s = 2^-delta s', t = 2^-delta (t' - delta s').
constexpr float kNear = 1048576.f;
__device__ __forceinline__ bool near_frame(float M) { return fabsf(M) <= kNear; }
__device__ __forceinline__ float frame_off(float m, float c) { return near_frame(m * c) ? fmaf(m, c, -(m * c)) : 0.f; }

// A lane's sums, in two pairs to shorten the chains of additions; kT: with sum 2^d d.  They are in the near
// frame of m where it has one, else relative to m itself.
template <bool kT>
struct LaneStat {
    float m;
    float2 s0, s1, t0, t1;
    __device__ __forceinline__ LaneStat() : m(-INFINITY) { s0 = s1 = t0 = t1 = make_float2(0.f, 0.f); }

    __device__ __forceinline__ void scale(float f, float d) {  // s <- f s, t <- f (t + d s)
        const float2 f2 = make_float2(f, f), d2 = make_float2(d, d);
        if (kT) {
            t0 = __fmul2_rn(f2, __ffma2_rn(d2, s0, t0));
            t1 = __fmul2_rn(f2, __ffma2_rn(d2, s1, t1));
        }
        s0 = __fmul2_rn(f2, s0);
        s1 = __fmul2_rn(f2, s1);
    }
    __device__ __forceinline__ void take(const LaneStat& b, float f, float d) {  // the same, and b's are added
        const float2 f2 = make_float2(f, f), d2 = make_float2(d, d);
        if (kT) {
            t0 = __ffma2_rn(f2, __ffma2_rn(d2, s0, t0), b.t0);
            t1 = __ffma2_rn(f2, __ffma2_rn(d2, s1, t1), b.t1);
        }
        s0 = __ffma2_rn(f2, s0, b.s0);
        s1 = __ffma2_rn(f2, s1, b.s1);
    }
    __device__ __forceinline__ void add(float2 d, int i) {
        const float2 e = make_float2(ex2(d.x), ex2(d.y));
        float2 &s = i & 1 ? s1 : s0, &t = i & 1 ? t1 : t0;
        s = __fadd2_rn(s, e);
        if (kT) t = __ffma2_rn(e, d, t);
    }

    // N units (of every lane of the warp) whose greatest logit is bm.
    template <bool kBf16, int N>
    __device__ __forceinline__ void add_units(const uint4 (&v)[N], float bm, float c) {
        const float nm = fmaxf(m, bm), Mo = m * c, M = nm * c;
        const float2 c2 = make_float2(c, c);
        LaneStat b;  // the sums of these units alone
        const bool far = !near_frame(M) || (!near_frame(Mo) && Mo > M + kCut);
        if (!__any_sync(0xffffffffu, far)) {
            const float2 nM = make_float2(-M, -M);
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < (kBf16 ? 4 : 2); ++i) b.add(__ffma2_rn(pair<kBf16>(v[k], i), c2, nM), i);
            // 2^d d of a masked token is 0 * -inf here: NaN says to take the longer way
            if (!kT || !__any_sync(0xffffffffu, isnan((b.t0.x + b.t0.y) + (b.t1.x + b.t1.y)))) {
                const float dm = fmaxf(Mo - M, kCut);
                take(b, ex2(dm), dm);
                m = nm;
                return;
            }
            b = LaneStat();
        }
        const float before = frame_off(m, c), after = frame_off(nm, c), p = pivot(nm);
        scale(ex2(-before), -before);
        const float dm = max_nan((m - p) * c, kCut);
        const float2 np = make_float2(-p, -p);
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < (kBf16 ? 4 : 2); ++i) {
                float2 d = __fmul2_rn(__fadd2_rn(pair<kBf16>(v[k], i), np), c2);
                d.x = max_nan(d.x, kCut);
                d.y = max_nan(d.y, kCut);
                b.add(d, i);
            }
        take(b, ex2(dm), dm);
        m = nm;
        scale(ex2(after), after);
    }

    __device__ __forceinline__ RowStat row(float c) {
        const float off = frame_off(m, c);
        scale(ex2(-off), -off);
        return RowStat{m, (s0.x + s0.y) + (s1.x + s1.y), (t0.x + t0.y) + (t1.x + t1.y)};
    }
};

// A part of a row has been written (by the whole warp): whether it is the last of the row's n, by a counter that is zero
// between launches.  The shuffle that tells the lanes orders no memory: what lets them read the other warps' parts is the
// barrier behind it, after lane 0's fence.
__device__ __forceinline__ bool arrive(uint32_t* count, int n) {
    uint32_t last = 0;
    __syncwarp();
    if ((threadIdx.x & 31) == 0) {
        __threadfence();
        last = atomicAdd(count, 1u) == (uint32_t)n - 1 ? 1u : 0u;
        if (last) *count = 0;
        __threadfence();
    }
    last = __shfl_sync(0xffffffffu, last, 0);
    __syncwarp();
    return last != 0;
}

// A unit whose elements from `valid` on are -inf: they count nowhere.
template <bool kBf16>
__device__ __forceinline__ void mask_unit(uint4& v, int valid) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int e = 0; e < (kBf16 ? 8 : 4); ++e)
        if (e >= valid) {
            if (!kBf16) w[e] = 0xFF800000u;
            else if (e & 1) w[e >> 1] = (w[e >> 1] & 0x0000FFFFu) | 0xFF800000u;
            else w[e >> 1] = (w[e >> 1] & 0xFFFF0000u) | 0x0000FF80u;
        }
}

template <bool kBf16>
__device__ __forceinline__ uint4 masked_unit() {
    const uint32_t w = kBf16 ? 0xFF80FF80u : 0xFF800000u;
    return make_uint4(w, w, w, w);
}

// A 16-byte load past L1 of memory that the kernel may write as well (ld_stream's must not be: a gradient may take
// its logits' place).
__device__ __forceinline__ uint4 ld_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

// Batches of a warp's next row that it asks for, into L2, when it is through with the one before: the join of a row takes
// microseconds in which it has no loads in flight.  Log probabilities of 30000 rows of 4000 tokens 87 -> 79 us, of 8192 of
// 32000 95 -> 93.5, of 4096 of 128256 165.5 -> 164 (cold L2; 2 and 4 batches alike, 16 worse for 32000; prefetches within a
// row cost, 170 and more for the last).
constexpr int kVocabAhead = 6;

// Units [c, c + n) of a row that end at c1 are on their way into L2 (a warp; one instruction of one lane).
__device__ __forceinline__ void fetch_units(const char* row, int c, int n, int c1) {
    n = min(n, c1 - c);
    if ((threadIdx.x & 31) == 0 && n > 0)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row + (int64_t)c * 16), "r"(n * 16) : "memory");
}

// The first units of the row behind `row` where a piece of the flat run goes on to `end` from u, that row's first unit.
__device__ __forceinline__ void fetch_next(const VocabRows& a, const char* row, int64_t u, int64_t end) {
    if (u < end) fetch_units(row + a.ld_bytes, 0, kVocabAhead * 32 * kVocabUnroll, (int)min(end - u, (int64_t)a.nvec));
}

// Unit c of a row whose units end at c1; past it, and past V, -inf.
template <bool kBf16>
__device__ __forceinline__ uint4 load_unit(const char* row, int c, int c1, int V) {
    constexpr int per = kBf16 ? 8 : 4;
    if (c >= c1) return masked_unit<kBf16>();
    uint4 v = ld_once(row + (int64_t)c * 16);
    if (V - c * per < per) mask_unit<kBf16>(v, V - c * per);
    return v;
}

// Element e of a unit, as fp32.
template <bool kBf16>
__device__ __forceinline__ float element(const uint4& v, int e) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
    if (!kBf16) return __uint_as_float(w[e]);
    return e & 1 ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
}

// The same where e is not known to the compiler.
template <bool kBf16>
__device__ __forceinline__ float element_of(const uint4& v, int e) {
    const int i = kBf16 ? e >> 1 : e;
    const uint32_t lo = i & 1 ? v.y : v.x, hi = i & 1 ? v.w : v.z, w = i & 2 ? hi : lo;
    if (!kBf16) return __uint_as_float(w);
    return e & 1 ? bf16hi(w) : bf16lo(w);
}

template <bool kBf16>
__device__ __forceinline__ float logit_at(const char* row, int v) {
    if (kBf16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[v]);
    return reinterpret_cast<const float*>(row)[v];
}

// A unit from fp32 values.
template <bool kBf16>
__device__ __forceinline__ void store_whole(char* p, const float (&x)[8]) {
    uint4 o;
    if (kBf16) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
    } else {
        o = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __stcs(reinterpret_cast<uint4*>(p), o);
}

// Unit c of a row of V.
template <bool kBf16>
__device__ __forceinline__ void store_unit(char* row, int c, int V, const float (&x)[8]) {
    constexpr int per = kBf16 ? 8 : 4;
    char* p = row + (int64_t)c * 16;
    if (V - c * per >= per) {
        store_whole<kBf16>(p, x);
    } else {  // the row's last, partial unit: what lies behind the vocabulary stays as it is
#pragma unroll
        for (int e = 0; e < per; ++e)
            if (c * per + e < V) {
                if (kBf16) reinterpret_cast<__nv_bfloat16*>(p)[e] = __float2bfloat16_rn(x[e]);
                else reinterpret_cast<float*>(p)[e] = x[e];
            }
    }
}

}  // namespace estp
