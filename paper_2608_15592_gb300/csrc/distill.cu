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
// A block takes a row: named units are marked in a bitmap, the statistics are taken in a first pass,
// one warp forms the loss and the row's factors, and the gradient is written in a second pass,
// whose reads come from L2.
#include "vocab.cuh"

namespace estp {
namespace {

constexpr int kDistillThreads = 512;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kSpanUnits = 1 << 16;  // units of a row that the bitmap covers at a time (8 KB)
constexpr int kK = kMaxAlternatives;

struct DistillArgs {
    const char* base;
    int64_t ld_bytes;
    int64_t n_rows;
    int32_t V, nvec;
    const int32_t* ids;
    const float* teacher;
    int K, tail;
    float T, c;
    const float* weight;
    float* loss;
    char* out;
    int64_t out_bytes;
    int* status;
};

struct DistillShared {
    uint32_t bits[kSpanUnits / 32];
    int32_t id[kK];
    float lq[kK], q[kK], z[kK], fix[kK];  // ln q, q, the student's logit, the gradient
    RowStat part[kDistillWarps];
    float A, pivot, Q, rest;
    int some;
};

template <class F>
__device__ __forceinline__ float warp_reduce(float x, F f) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x = f(x, __shfl_xor_sync(0xffffffffu, x, off));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
    return warp_reduce(x, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// The teacher's side of a row (one warp): q and ln q of the named tokens, the rest, and the student's
// logits there.
template <bool kBf16>
__device__ void teacher_row(const DistillArgs& a, int64_t r, DistillShared& s) {
    const int lane = threadIdx.x & 31;
    const char* row = a.base + r * a.ld_bytes;
    float x[kK / 32], top = -INFINITY;
    bool some = false;
#pragma unroll
    for (int i = 0; i < kK / 32; ++i) {
        const int j = i * 32 + lane;
        x[i] = -INFINITY;
        if (j < a.K && s.id[j] >= 0) {
            x[i] = a.teacher[r * a.K + j];
            s.z[j] = logit_at<kBf16>(row, s.id[j]);
            some = true;
        }
        top = fmaxf(top, x[i]);
    }
    float Q, rest = 0.f;
    some = __any_sync(0xffffffffu, some);
    if (a.tail) {
        double sum = 0.;
#pragma unroll
        for (int i = 0; i < kK / 32; ++i) {
            const int j = i * 32 + lane;
            const float q = expf(x[i]);
            sum += (double)q;
            if (j < a.K) {
                s.q[j] = q;
                s.lq[j] = x[i];
            }
        }
        sum = warp_sum(sum);
        Q = (float)sum;
        rest = !some || sum > 1. ? 0.f : (float)(1. - sum);
    } else {
        top = pivot(warp_reduce(top, [](float p, float q) { return fmaxf(p, q); }));
        float e[kK / 32], sum = 0.f;
#pragma unroll
        for (int i = 0; i < kK / 32; ++i) {
            e[i] = expf((x[i] - top) / a.T);
            sum += e[i];
        }
        sum = warp_sum(sum);
        const bool none = sum == 0.f;  // every entry of -inf: no teacher
        const float l = none ? 0.f : logf(sum);
#pragma unroll
        for (int i = 0; i < kK / 32; ++i) {
            const int j = i * 32 + lane;
            if (j < a.K) {
                s.q[j] = none ? 0.f : e[i] / sum;
                s.lq[j] = (x[i] - top) / a.T - l;
            }
        }
        Q = none ? 0.f : 1.f;
        some = !none;
    }
    if (lane == 0) {
        s.Q = Q;
        s.rest = rest;
        s.some = some;
    }
}

// The loss and the row's factors (one warp), from the statistics `st` of every token, or with the tail
// of the tokens that are not named.
__device__ void finish_row(const DistillArgs& a, int64_t r, DistillShared& s, const RowStat& st, float g) {
    const int lane = threadIdx.x & 31;
    const float Q = s.Q;
    float rest = s.rest;
    // Where the student has no other token, what the teacher leaves to them may be the rounding of its log
    // probabilities: sum q_j |x_j| 2^-24 + 2^-23 at most, below 2^-20 for the entropies that 128 tokens have.
    const bool no_other = st.s == 0.f;
    if (a.tail && no_other && rest <= 0x1p-20f) rest = 0.f;
    RowStat all = st;
    if (a.tail) {
        RowStat in = no_stat();
#pragma unroll
        for (int i = 0; i < kK / 32; ++i) {
            const int j = i * 32 + lane;
            if (j < a.K && s.id[j] >= 0) join(in, RowStat{s.z[j], isnan(s.z[j]) || s.z[j] == INFINITY ? NAN : s.z[j] == -INFINITY ? 0.f : 1.f, 0.f}, a.c);
        }
        join_lanes(in, a.c);
        join(all, in, a.c);
    }
    const bool empty = all.s == 0.f;
    const float m = pivot(all.m), ls = empty ? -INFINITY : logf(all.s);
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < kK / 32; ++i) {
        const int j = i * 32 + lane;
        if (j < a.K && s.id[j] >= 0) {
            const float q = s.q[j], lp = empty ? -INFINITY : (s.z[j] - m) / a.T - ls;
            // q first: beside a logit of the type's lowest value ln p may exceed fp32 where the loss does not
            if (q != 0.f) loss += empty ? INFINITY : q * (s.lq[j] + ls) + q * (m - s.z[j]) / a.T;
            if (a.tail) s.fix[j] = empty ? 0.f : g * ((Q + rest) * expf(lp) - q);
            else s.fix[j] = empty ? 0.f : -g * q;
        }
    }
    loss = warp_sum(loss);
    // the exponentials of the second pass are taken against the maximum that its sums belong to
    float A = empty ? 0.f : g * (Q + rest) / all.s;
    if (a.tail) {
        const float mo = pivot(st.m);
        if (rest != 0.f) loss += rest * (logf(rest) - (no_other || empty ? -INFINITY : (mo - m) / a.T + (logf(st.s) - ls)));
        A = no_other || empty ? 0.f : g * ((Q + rest) * ex2(max_nan((mo - m) * a.c, kCut)) / all.s - rest / st.s);
        if (lane == 0) s.pivot = mo;
    } else if (lane == 0) {
        s.pivot = m;
    }
    if (lane == 0) {
        s.A = A;
        a.loss[r] = s.some ? loss : 0.f;
    }
}

// Calls f(j) in every lane for each named token j of the unit that lane `f_lane` holds.
template <class F>
__device__ __forceinline__ void each_named(const DistillShared& s, int K, int per, int unit, F f) {
    const int lane = threadIdx.x & 31;
    for (int i0 = 0; i0 < K; i0 += 32) {
        const int i = i0 + lane;
        const int id = i < K ? s.id[i] : -1;
        uint32_t hit = __ballot_sync(0xffffffffu, id >= 0 && id / per == unit);
        while (hit) {
            const int j = i0 + __ffs(hit) - 1;
            hit &= hit - 1;
            f(j);
        }
    }
}

template <bool kBf16>
__device__ __forceinline__ void mask_element(uint4& v, int at) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int e = 0; e < (kBf16 ? 8 : 4); ++e)
        if (e == at) {
            if (!kBf16) w[e] = 0xFF800000u;
            else if (e & 1) w[e >> 1] = (w[e >> 1] & 0x0000FFFFu) | 0xFF800000u;
            else w[e >> 1] = (w[e >> 1] & 0xFFFF0000u) | 0x0000FF80u;
        }
}

// Marks (or clears) the units of [span, span + kSpanUnits) that hold a named token.
__device__ __forceinline__ void mark(const DistillArgs& a, DistillShared& s, int per, int span, bool set) {
    for (int j = threadIdx.x; j < a.K; j += kDistillThreads) {
        const unsigned k = (unsigned)(s.id[j] / per - span);
        if (s.id[j] >= 0 && k < (unsigned)kSpanUnits) {
            if (set) atomicOr(&s.bits[k >> 5], 1u << (k & 31));
            else s.bits[k >> 5] = 0;
        }
    }
}

template <bool kBf16>
__device__ __forceinline__ void store_row_unit(char* row, int c, int V, const float (&x)[8]) {
    constexpr int per = kBf16 ? 8 : 4;
    char* p = row + (int64_t)c * 16;
    if (V - c * per >= per) {
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
    } else {
#pragma unroll
        for (int e = 0; e < per; ++e)
            if (c * per + e < V) {
                if (kBf16) reinterpret_cast<__nv_bfloat16*>(p)[e] = __float2bfloat16_rn(x[e]);
                else reinterpret_cast<float*>(p)[e] = x[e];
            }
    }
}

template <bool kBf16>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillArgs a) {
    constexpr int per = kBf16 ? 8 : 4, kStep = 32 * kVocabUnroll;
    __shared__ DistillShared s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < kSpanUnits / 32; i += kDistillThreads) s.bits[i] = 0;
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        if (!in_bounds(r >= 0 && a.nvec * (int64_t)per >= a.V, a.status)) return;
        const char* row = a.base + r * a.ld_bytes;
        __syncthreads();
        for (int j = tid; j < a.K; j += kDistillThreads) {
            int id = a.ids[r * a.K + j];
            if (id >= a.V) {
                report(a.status, ESTP_ERR_INVALID_ARG);
                id = -1;
            }
            s.id[j] = id;
        }
        __syncthreads();
        if (a.tail) {  // a token has one probability: a repeated one is left out
            for (int j = tid; j < a.K; j += kDistillThreads) {
                bool again = false;
                for (int i = 0; i < j; ++i) again |= s.id[i] == s.id[j];
                s.fix[j] = again && s.id[j] >= 0 ? 1.f : 0.f;
            }
            __syncthreads();
            for (int j = tid; j < a.K; j += kDistillThreads)
                if (s.fix[j] != 0.f) {
                    report(a.status, ESTP_ERR_INVALID_ARG);
                    s.id[j] = -1;
                }
            __syncthreads();
        }
        if (warp == 0) teacher_row<kBf16>(a, r, s);
        const float g = (a.weight ? a.weight[r] : 1.f) / a.T;
        // first pass: the statistics
        LaneStat st;
        const float2 c2 = make_float2(a.c, a.c);
        for (int span = 0; span < a.nvec; span += kSpanUnits) {
            const int stop = min(a.nvec, span + kSpanUnits);
            if (a.tail) {
                mark(a, s, per, span, true);
                __syncthreads();
            }
            for (int b = span + warp * kStep; b < stop; b += kDistillWarps * kStep) {
                uint4 v[kVocabUnroll];
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) v[k] = load_unit<kBf16>(row, b + 32 * k + lane, stop, a.V);
                if (a.tail) {
#pragma unroll
                    for (int k = 0; k < kVocabUnroll; ++k) {
                        const int c = b + 32 * k;
                        uint32_t lanes = c < stop ? s.bits[(c - span) >> 5] : 0;
                        while (lanes) {
                            const int f = __ffs(lanes) - 1;
                            lanes &= lanes - 1;
                            each_named(s, a.K, per, c + f, [&](int j) {
                                const int at = s.id[j] - (c + f) * per;
                                if (lane == f) mask_element<kBf16>(v[k], at);
                            });
                        }
                    }
                }
                float bm = unit_max<kBf16>(v[0]);
#pragma unroll
                for (int k = 1; k < kVocabUnroll; ++k) bm = fmaxf(bm, unit_max<kBf16>(v[k]));
                const float p = -st.raise(bm, a.c);
                const float2 np = make_float2(p, p);
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) add_unit<kBf16>(v[k], np, c2, st);
            }
            if (a.tail) {
                __syncthreads();
                mark(a, s, per, span, false);
                __syncthreads();
            }
        }
        RowStat mine = st.row();
        join_lanes(mine, a.c);
        if (lane == 0) s.part[warp] = mine;
        __syncthreads();
        if (warp == 0) {
            RowStat all = lane < kDistillWarps ? s.part[lane] : no_stat();
            join_lanes(all, a.c);
            finish_row(a, r, s, all, g);
        }
        __syncthreads();
        if (!a.out) continue;
        // second pass: the gradient
        char* out = a.out + r * a.out_bytes;
        const bool zero = !s.some || g == 0.f;
        const float2 np = make_float2(-s.pivot, -s.pivot);
        const float A = s.A;
        for (int span = 0; span < a.nvec; span += kSpanUnits) {
            const int stop = min(a.nvec, span + kSpanUnits);
            mark(a, s, per, span, true);
            __syncthreads();
            for (int b = span + warp * kStep; b < stop; b += kDistillWarps * kStep) {
                uint4 v[kVocabUnroll];
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) v[k] = load_unit<kBf16>(row, b + 32 * k + lane, stop, a.V);
#pragma unroll
                for (int k = 0; k < kVocabUnroll; ++k) {
                    const int c = b + 32 * k;
                    float x[8];
#pragma unroll
                    for (int e = 0; e < per; e += 2) {
                        const float2 d = __fmul2_rn(__fadd2_rn(make_float2(element<kBf16>(v[k], e), element<kBf16>(v[k], e + 1)), np), c2);
                        x[e] = zero ? 0.f : A * ex2(d.x);
                        x[e + 1] = zero ? 0.f : A * ex2(d.y);
                    }
                    uint32_t lanes = c < stop && !zero ? s.bits[(c - span) >> 5] : 0;
                    while (lanes) {
                        const int f = __ffs(lanes) - 1;
                        lanes &= lanes - 1;
                        each_named(s, a.K, per, c + f, [&](int j) {
                            const int at = s.id[j] - (c + f) * per;
#pragma unroll
                            for (int e = 0; e < per; ++e)
                                if (lane == f && e == at) x[e] = a.tail ? s.fix[j] : x[e] + s.fix[j];
                        });
                    }
                    if (c + lane < stop) store_row_unit<kBf16>(out, c + lane, a.V, x);
                }
            }
            __syncthreads();
            mark(a, s, per, span, false);
            __syncthreads();
        }
    }
}

}  // namespace

estp_status launch_distill_loss(estp_ctx* ctx, const void* logits, estp_dtype dtype, int64_t n_rows, int64_t V,
                                int64_t ld, const int32_t* ids, const float* teacher, int K, float T, bool tail,
                                const float* weight, float* loss, void* out, int64_t ld_out, cudaStream_t st) {
    DistillArgs a;
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
    a.weight = weight;
    a.loss = loss;
    a.out = static_cast<char*>(out);
    a.out_bytes = ld_out * esize(dtype);
    a.status = ctx->status;
    const int64_t most = (int64_t)ctx->num_sms * 2;
    const unsigned blocks = (unsigned)(n_rows < most ? n_rows : most);
    if (dtype == ESTP_BF16) distill_kernel<true><<<blocks, kDistillThreads, 0, st>>>(a);
    else distill_kernel<false><<<blocks, kDistillThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "distillation launch");
}

}  // namespace estp
