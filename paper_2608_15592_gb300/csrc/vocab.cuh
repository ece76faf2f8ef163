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
constexpr int kVocabBlocks = 3;       // resident blocks an SM the registers of the streams are sized for
constexpr int kVocabUnroll = 8;       // 16-byte loads a lane has in flight
constexpr int kMaxAlternatives = 128;  // entries of a row's list
constexpr int64_t kMaxVocab = 1 << 30;  // a token's index, and that of its unit, in 32 bits
constexpr float kMinTemperature = 1e-6f;  // log2(e) / T stays far from overflow
constexpr float kCut = -200.f;

__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// ------------------------------------------------------------------ the flat cut
// The rows as one run of 16-byte units, cut into equal pieces, a warp each: every warp streams the
// same number of bytes whatever V and n_rows are.
struct VocabRows {
    const char* base;
    int64_t ld_bytes;
    int64_t n_rows;
    int64_t units;   // n_rows * nvec
    int64_t pieces;
    int32_t V;
    int32_t nvec;    // units of a row (the last one may be partial)
};

__device__ __forceinline__ int64_t piece_start(const VocabRows& a, int64_t w) { return a.units * w / a.pieces; }

// The last piece that starts at or before unit u.
__device__ __forceinline__ int64_t piece_of(const VocabRows& a, int64_t u) {
    const int64_t w = ((u + 1) * a.pieces - 1) / a.units;
    return w < a.pieces - 1 ? w : a.pieces - 1;
}

inline VocabRows vocab_rows(const estp_ctx* ctx, const void* logits, estp_dtype dtype, int64_t n_rows, int64_t V,
                            int64_t ld, int min_units) {
    VocabRows a;
    const int per = 16 / esize(dtype);
    a.base = static_cast<const char*>(logits);
    a.ld_bytes = ld * esize(dtype);
    a.n_rows = n_rows;
    a.V = (int32_t)V;
    a.nvec = (int32_t)((V + per - 1) / per);
    a.units = n_rows * a.nvec;
    const int64_t most = (int64_t)ctx->num_sms * kVocabBlocks * (kVocabThreads / 32);
    const int64_t want = (a.units + min_units - 1) / min_units;
    a.pieces = want < most ? want : most;
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

__device__ __forceinline__ void join_lanes(RowStat& a, float c) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const RowStat b{__shfl_xor_sync(0xffffffffu, a.m, off), __shfl_xor_sync(0xffffffffu, a.s, off),
                        __shfl_xor_sync(0xffffffffu, a.t, off)};
        join(a, b, c);
    }
}

// A lane's sums, in two pairs to shorten the chains of additions.
struct LaneStat {
    float m;
    float2 s0, s1, t0, t1;
    __device__ __forceinline__ LaneStat() : m(-INFINITY) { s0 = s1 = t0 = t1 = make_float2(0.f, 0.f); }
    __device__ __forceinline__ RowStat row() const {
        return RowStat{m, (s0.x + s0.y) + (s1.x + s1.y), (t0.x + t0.y) + (t1.x + t1.y)};
    }
    // Sums in units of the new maximum; returns what is subtracted from the logits.
    __device__ __forceinline__ float raise(float bm, float c) {
        const float nm = fmaxf(m, bm), p = pivot(nm);
        const float dm = max_nan((m - p) * c, kCut), f = ex2(dm);
        const float2 f2 = make_float2(f, f), d2 = make_float2(dm, dm);
        t0 = __fmul2_rn(f2, __ffma2_rn(d2, s0, t0));
        t1 = __fmul2_rn(f2, __ffma2_rn(d2, s1, t1));
        s0 = __fmul2_rn(f2, s0);
        s1 = __fmul2_rn(f2, s1);
        m = nm;
        return p;
    }
};

__device__ __forceinline__ void add_pair(float x, float y, float2 np, float2 c2, float2& s, float2& t) {
    float2 d = __fmul2_rn(__fadd2_rn(make_float2(x, y), np), c2);
    d.x = max_nan(d.x, kCut);
    d.y = max_nan(d.y, kCut);
    const float2 e = make_float2(ex2(d.x), ex2(d.y));
    s = __fadd2_rn(s, e);
    t = __ffma2_rn(e, d, t);
}

template <bool kBf16>
__device__ __forceinline__ void add_unit(const uint4& v, float2 np, float2 c2, LaneStat& a) {
    if (kBf16) {
        add_pair(bf16lo(v.x), bf16hi(v.x), np, c2, a.s0, a.t0);
        add_pair(bf16lo(v.y), bf16hi(v.y), np, c2, a.s1, a.t1);
        add_pair(bf16lo(v.z), bf16hi(v.z), np, c2, a.s0, a.t0);
        add_pair(bf16lo(v.w), bf16hi(v.w), np, c2, a.s1, a.t1);
    } else {
        add_pair(__uint_as_float(v.x), __uint_as_float(v.y), np, c2, a.s0, a.t0);
        add_pair(__uint_as_float(v.z), __uint_as_float(v.w), np, c2, a.s1, a.t1);
    }
}

// Greatest logit of a unit (NaN is passed over: the sums show it).
template <bool kBf16>
__device__ __forceinline__ float unit_max(const uint4& v) {
    if (kBf16) {
        const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 x = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        return fmaxf(__low2float(x), __high2float(x));
    }
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
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

// Unit c of a row whose units end at c1; past it, and past V, -inf.
template <bool kBf16>
__device__ __forceinline__ uint4 load_unit(const char* row, int c, int c1, int V) {
    constexpr int per = kBf16 ? 8 : 4;
    if (c >= c1) return masked_unit<kBf16>();
    uint4 v = ld_stream(row + (int64_t)c * 16);
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

template <bool kBf16>
__device__ __forceinline__ float logit_at(const char* row, int v) {
    if (kBf16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[v]);
    return reinterpret_cast<const float*>(row)[v];
}

}  // namespace estp
