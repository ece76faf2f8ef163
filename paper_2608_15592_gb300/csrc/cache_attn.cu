// Attention of a step's rows over a paged KV cache, with the attention weight that every cached
// slot receives:
//   s_ij = scale q_i . k_j,  lse_i = ln sum_j e^s_ij,  o_i = sum_j e^(s_ij - lse_i) v_j,
//   weight_j += sum_i c_i e^(s_ij - lse_i)
// over the cached slots and the drafts that row i sees:
//
// cache_fwd_kernel: a persistent grid over the units of cache.cuh.  Of every group segment it
// leaves the running maximum m (log2 units), the sum l = sum 2^(s' - m) and O = sum 2^(s' - m) v,
// s' = s log2(e), and, where the weights are wanted and fit, every unscaled score q.k.
//
// cache_finish_kernel: merges the partials of each row in CTA order, writes o and lse, and adds to
// every slot the weight of its rows, sum_r c_r 2^(s' - M_r) / L_r, from the kept scores.  With many
// rows to a key, keeping scores costs more than forming them again: cache_weight_kernel does, a
// third launch.  No floating-point atomics: every sum has one order.
//
// The finish is bound by latency when there are few rows (4 to 7 us), by its bytes with many sequences: a
// tile of 4 rows and 128 keys is 2 KB of scores beside 1 KB of weights, read and written.
//
// A row that sees nothing (M = -inf, L = 0) gives o = 0 and lse = -inf and no weight.
//
// Weights cannot be formed a second time: after a wait that ran out nothing is added to them, by this call
// or a later one, until the program has read the status.
#include "cache_tc.cuh"

namespace estp {
namespace {

constexpr int kThreads = 128;  // one key of a tile each
constexpr int kRows = 8;       // rows of a block of the CUDA-core kernels
constexpr int kBlocks = 3;     // of those an SM: 168 registers a thread (4 blocks: 79 us where 3 take 66, as below)
constexpr int kCacheMaxStored = 64;  // rows of a (b, KV head) whose scores are kept at most

template <class T> struct Unit;  // 16 bytes of a row
template <> struct Unit<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const char* p, float* v) {
        const float4 x = *reinterpret_cast<const float4*>(p);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    }
    static __device__ __forceinline__ float one(const char* p) { return *reinterpret_cast<const float*>(p); }
    static __device__ __forceinline__ void put(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
};
template <> struct Unit<__nv_bfloat16> {
    static __device__ __forceinline__ void get(const char* p, float* v) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        v[0] = bf16lo(x.x); v[1] = bf16hi(x.x); v[2] = bf16lo(x.y); v[3] = bf16hi(x.y);
        v[4] = bf16lo(x.z); v[5] = bf16hi(x.z); v[6] = bf16lo(x.w); v[7] = bf16hi(x.w);
    }
    static __device__ __forceinline__ float one(const char* p) {
        return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
    }
    static __device__ __forceinline__ void put(char* p, float v) {
        *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
    }
};

// Where key j of a tile lies: NULL past the tile's keys (or on a page that is none).
struct KeyRow {
    const char* k;
    const char* v;
    int64_t meta;  // weight element of a cached slot
};
__device__ __forceinline__ KeyRow key_row(const CacheAttnArgs& a, const SeqShape& q, int b, int g, int tile, int j,
                                          int row_bytes) {
    KeyRow r{nullptr, nullptr, -1};
    if (tile == q.nt - 1) {
        if (a.kn != nullptr && j < q.n) {
            const int64_t off = (int64_t)(a.cu[b] + j) * a.ldn + (int64_t)g * row_bytes;
            r.k = a.kn + off;
            r.v = a.vn + off;
        }
    } else {
        const int slot = tile * kCacheTile + j;
        if (slot < q.len) {
            const int64_t page = a.c.page_of(b, slot, a.status);
            if (page >= 0) {
                const int64_t off = a.c.row(page, slot, g);
                r.k = a.c.k + off;
                r.v = a.c.v + off;
                r.meta = a.c.meta(page, slot, g);
            }
        }
    }
    return r;
}

// kRows rows of Q, from row r0 of (b, g), as floats; rows past nr are zero.
template <class T, int D>
__device__ __forceinline__ void load_q(const CacheAttnArgs& a, float (*q)[D], int b, int g, int r0, int nr) {
    constexpr int kU = D / Unit<T>::n;
    for (int e = threadIdx.x; e < kRows * kU; e += kThreads) {
        const int r = e / kU, c = e % kU;
        float v[Unit<T>::n];
        for (int i = 0; i < Unit<T>::n; ++i) v[i] = 0.f;
        if (r < nr) {
            const int i = (r0 + r) / a.rep, h = g * a.rep + (r0 + r) % a.rep;
            Unit<T>::get(a.Q + (a.cu[b] + i) * a.ldq + ((int64_t)h * D) * sizeof(T) + c * 16, v);
        }
        for (int i = 0; i < Unit<T>::n; ++i) q[r][c * Unit<T>::n + i] = v[i];
    }
}

// z[r] = q_r . k, k the calling thread's key row (NULL: 0), by a whole warp for its 32 keys: 8 lanes read
// a row together, 128 bytes at a time (a lane a row touches as many cache lines as lanes an instruction:
// 103 us for 5 drafts and 8 query heads a KV head over 20000 fp32 tokens of 2 x 128, 66 so), and 4 keys a
// lane share each read of q.  zs: the warp's 32 rows of scratch.
template <int D>
__device__ __forceinline__ void dots(const float (*q)[D], const char* k, float (*zs)[kRows], float* z) {
    static_assert(kRows == 8, "8 lanes a key, a row each at the end");
    constexpr int kPer = 4;
    const int lane = threadIdx.x & 31, sub = lane & 7, grp = lane >> 3;
#pragma unroll 1
    for (int k0 = 0; k0 < 32; k0 += 4 * kPer) {
        const char* kp[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            kp[i] = reinterpret_cast<const char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(k), k0 + 4 * i + grp));
        float2 acc[kPer][kRows] = {};  // even and odd dimensions: packed FMAs
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            float4 kv[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                kv[i] = kp[i] != nullptr ? *reinterpret_cast<const float4*>(kp[i] + (c * 8 + sub) * 16) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(&q[r][(c * 8 + sub) * 4]);
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    acc[i][r] = __ffma2_rn(make_float2(x.x, x.y), make_float2(kv[i].x, kv[i].y), acc[i][r]);
                    acc[i][r] = __ffma2_rn(make_float2(x.z, x.w), make_float2(kv[i].z, kv[i].w), acc[i][r]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {  // over the 8 lanes: each step halves the rows a lane still holds
            float v[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) v[r] = acc[i][r].x + acc[i][r].y;
#pragma unroll
            for (int o = kRows / 2; o > 0; o >>= 1)
#pragma unroll
                for (int r = 0; r < o; ++r) {
                    const bool up = sub & o;
                    v[r] = (up ? v[r + o] : v[r]) + __shfl_xor_sync(0xffffffffu, up ? v[r] : v[r + o], o);
                }
            zs[k0 + 4 * i + grp][sub] = v[0];
        }
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < kRows; r += 4) {
        const float4 x = *reinterpret_cast<const float4*>(&zs[lane][r]);
        z[r] = x.x; z[r + 1] = x.y; z[r + 2] = x.z; z[r + 3] = x.w;
    }
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, kBlocks) cache_fwd_kernel(const CacheAttnArgs a) {
    __shared__ PlanScratch sc;
    __shared__ __align__(16) float q[kRows][D];
    __shared__ __align__(16) float p[kCacheTile][kRows];
    __shared__ const char* vrow[kCacheTile];
    __shared__ float red[kThreads / 32][kRows];
    __shared__ float o_half[kRows][D];
    await_stream();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int c = blockIdx.x;
    Place at;
    const PlanTotals tot = plan(a, &sc, &at, [&](const Place& x, const SeqShape& s, const PlanTotals& all) {
        const int u = share_begin(c, all.units, ctas_of(a, all.units));
        return u >= x.unit0 && u < x.unit0 + s.units(a.c.Hkv);
    });
    const int G = ctas_of(a, tot.units);
    if (!tot.ok || c >= G) return;
    int u = share_begin(c, tot.units, G);
    const int u1 = share_begin(c + 1, tot.units, G);
    constexpr int kHalves = kThreads / D, kKeys = kCacheTile / kHalves;  // PV: threads of a column, keys of each
    const int col = t % D, half = t / D;
    while (u < u1) {
        const SeqShape s = seq_shape(a, at.b);
        if (u >= at.unit0 + s.units(a.c.Hkv)) {
            at.pass(s, a.c.Hkv);
            continue;
        }
        const Span span = span_of(a, s, u - at.unit0, u1 - u);
        const int g = span.g, grp = g * s.nrb + span.k, tile0 = span.tile0, tile1 = span.tile1;
        const int r0 = span.k * kRows, nr = min(kRows, s.n * a.rep - r0);
        const int64_t row0 = a.cu[at.b];
        __syncthreads();
        load_q<T, D>(a, q, at.b, g, r0, nr);
        float m[kRows], l[kRows];
        float2 o[kRows / 2] = {};  // two rows each
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
        }
        for (int tile = tile0; tile < tile1; ++tile, ++u) {
            const bool drafts = tile == s.nt - 1;
            const KeyRow kr = key_row(a, s, at.b, g, tile, t, D * (int)sizeof(T));
            __syncthreads();  // p and vrow are free, q is there
            float z[kRows];
            dots<D>(q, kr.k, p + warp * 32, z);  // p is free: every thread overwrites its own row
            vrow[t] = kr.v;
            unsigned hidden = 0;  // rows that do not see this key
            if (drafts) {
                hidden = ~(unsigned)rows_that_see(a, row0, kr.k != nullptr ? s.n : 0, t, r0, nr);
            } else if (kr.k == nullptr) {
                hidden = (1u << kRows) - 1;
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (hidden >> r & 1) z[r] = -INFINITY;
            if (a.store && a.unit_inside(u))
                for (int r = 0; r < nr; ++r) a.score[((int64_t)u * kRows + r) * kCacheTile + t] = z[r];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                float x = z[r];
                for (int w = 16; w > 0; w >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
                if (lane == 0) red[warp][r] = x;
            }
            __syncthreads();
            float pr[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const float top = fmaxf(fmaxf(red[0][r], red[1][r]), fmaxf(red[2][r], red[3][r])) * a.scale_log2;
                const float mn = fmaxf(m[r], top);
                const float f = m[r] == mn ? 1.f : ex2(m[r] - mn);  // m = -inf: 0, and l = o = 0
                m[r] = mn;
                const float e = ex2(fmaf(z[r], a.scale_log2, mn == -INFINITY ? 0.f : -mn));
                l[r] = fmaf(l[r], f, hidden >> r & 1 ? 0.f : e);
                (r & 1 ? o[r / 2].y : o[r / 2].x) *= f;
                pr[r] = hidden >> r & 1 ? (drafts ? -1.f : 0.f) : e;  // -1: no probability, the draft is left out
            }
#pragma unroll
            for (int r = 0; r < kRows; r += 4) *reinterpret_cast<float4*>(&p[t][r]) = make_float4(pr[r], pr[r + 1], pr[r + 2], pr[r + 3]);
            __syncthreads();
            constexpr int kBatch = 16;  // V rows in flight
            for (int j0 = half * kKeys; j0 < (half + 1) * kKeys; j0 += kBatch) {
                float v[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const char* vr = vrow[j0 + k];
                    v[k] = vr != nullptr ? Unit<T>::one(vr + col * sizeof(T)) : 0.f;
                }
                if (!drafts) {
#pragma unroll
                    for (int k = 0; k < kBatch; ++k)
#pragma unroll
                        for (int r = 0; r < kRows; r += 4) {
                            const float4 e = *reinterpret_cast<const float4*>(&p[j0 + k][r]);
                            const float2 v2 = make_float2(v[k], v[k]);
                            o[r / 2] = __ffma2_rn(make_float2(e.x, e.y), v2, o[r / 2]);
                            o[r / 2 + 1] = __ffma2_rn(make_float2(e.z, e.w), v2, o[r / 2 + 1]);
                        }
                } else {  // what a hidden draft's V holds adds nothing, 0 x NaN included
#pragma unroll
                    for (int k = 0; k < kBatch; ++k)
#pragma unroll
                        for (int r = 0; r < kRows; ++r) {
                            const float e = p[j0 + k][r];
                            float& x = r & 1 ? o[r / 2].y : o[r / 2].x;
                            if (!(e < 0.f)) x = fmaf(e, v[k], x);
                        }
                }
            }
        }
        // the segment's partial: l over the keys' threads, O over the halves
        const int64_t slot = c + at.group0 + grp;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float x = l[r];
            for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
            if (lane == 0) red[warp][r] = x;
            if (half == 1) o_half[r][col] = r & 1 ? o[r / 2].y : o[r / 2].x;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r >= nr || !a.part_inside(slot)) break;
            if (t == 0)
                a.part_ml[slot * kRows + r] = make_float2(m[r], (red[0][r] + red[1][r]) + (red[2][r] + red[3][r]));
            const float x = r & 1 ? o[r / 2].y : o[r / 2].x;
            if (half == 0) a.part_o[(slot * kRows + r) * D + col] = kHalves == 2 ? x + o_half[r][col] : x;
        }
    }
    admit_next();
}

// Pieces of row r of (b, g): CTAs c0..c1 hold the group, each with a partial at slot c + group.
struct Pieces {
    int64_t first;  // part_ml element of the first
    int n;          // the others RB apart
};
__device__ __forceinline__ Pieces pieces_of(const CacheAttnArgs& a, const Place& at, const SeqShape& s, int g, int r,
                                            int units) {
    const int k = r / a.RB, per = a.RB > 128 ? 2 : 1, grp = g * s.nrb + k, G = ctas_of(a, units);
    const int ub = at.unit0 + (g * s.cost + k * per) * s.nt;
    const int c0 = share_of(ub, units, G), c1 = share_of(ub + (k < s.nrb - 1 ? per : s.last) * (s.nt - 1), units, G);
    return Pieces{(int64_t)(c0 + at.group0 + grp) * a.RB + r % a.RB, c1 - c0 + 1};
}

// Joins (M, L) with another running maximum and sum.  Unfused products: two lanes that join each
// other's get the same bits.
__device__ __forceinline__ void merge_ml(float& M, float& L, float2 x) {
    const float mn = fmaxf(M, x.x);
    // -inf on both sides: nothing was summed, or NaN, which stays
    if (mn != -INFINITY) L = __fadd_rn(__fmul_rn(L, ex2(M - mn)), __fmul_rn(x.y, ex2(x.x - mn)));
    else L += x.y;
    M = mn;
}

// Warp-wide: the row's maximum and sum over its pieces.
__device__ __forceinline__ float2 merged_ml(const CacheAttnArgs& a, const Pieces& w, int lane) {
    float M = -INFINITY, L = 0.f;
    for (int c = lane; c < w.n; c += 32) merge_ml(M, L, a.part_ml[w.first + (int64_t)c * a.RB]);
    for (int o = 16; o > 0; o >>= 1)
        merge_ml(M, L, make_float2(__shfl_xor_sync(0xffffffffu, M, o), __shfl_xor_sync(0xffffffffu, L, o)));
    return make_float2(M, L);
}

// Walks a CTA's share [it, it1) of the call's items (b, KV head, tile) in runs of one (b, KV head).
template <class Run>
__device__ __forceinline__ void for_items(const CacheAttnArgs& a, Place at, int it, int it1, Run run) {
    while (it < it1) {
        const SeqShape s = seq_shape(a, at.b);
        if (it >= at.item0 + s.items(a.c.Hkv)) {
            at.pass(s, a.c.Hkv);
            continue;
        }
        const int g = (it - at.item0) / s.nt, tile0 = (it - at.item0) % s.nt;
        const int tile1 = min(s.nt, tile0 + (it1 - it));
        run(at, s, g, tile0, tile1);
        it += tile1 - tile0;
    }
}

// The first a.row_blocks blocks merge the partials: o and lse, a warp or a block a (row, head), cut
// evenly over them; without kept scores they leave (-M, c / L) of every row for the kernel that forms the scores
// again.  With kept scores the other blocks add the weights, the (b, KV head, tile) items cut evenly
// over their warps: a warp a tile, a lane 4 keys.
template <class T, int D>
__global__ void __launch_bounds__(kThreads, 8) cache_finish_kernel(const CacheAttnArgs a) {
    __shared__ PlanScratch sc;
    __shared__ float2 ml[kThreads / 32][kCacheMaxStored];  // a warp's (-M, c / L) of every row of (b, g)
    admit_next();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const bool for_rows = (int)blockIdx.x < a.row_blocks;
    const int c = for_rows ? blockIdx.x : blockIdx.x - a.row_blocks;
    const int G = for_rows ? a.row_blocks : gridDim.x - a.row_blocks, rows = (int)a.n_rows * a.Hq;
    const int x0 = share_begin(c, rows, G), x1 = share_begin(c + 1, rows, G);
    Place at;
    const PlanTotals tot = plan(a, &sc, &at, [&](const Place& x, const SeqShape& s, const PlanTotals& all) {
        const int y = a.cu[x.b] * a.Hq, it = share_begin(c, all.items, G);
        return for_rows ? x0 >= y && x0 < y + s.n * a.Hq : it >= x.item0 && it < x.item0 + s.items(a.c.Hkv);
    });
    await_stream();  // the partials are complete
    const bool lost = *a.timed_out != 0;  // or a wait ran out, and nothing is added from what they happen to hold
    if (!tot.ok) return;
    if (for_rows) {
        if (x0 >= x1) return;
        __shared__ float part[kThreads / 32][D];
        constexpr int kC = D / 32;
        SeqShape s = seq_shape(a, at.b);
        const int wide = a.row_warps;  // warps of a row: they take its pieces in turn, 8 in flight, and are added in order
        for (int x = x0 + (wide == 1 ? warp : 0); x < x1; x += wide == 1 ? kThreads / 32 : 1) {
            while (x >= a.cu[at.b + 1] * a.Hq) {
                at.pass(s, a.c.Hkv);
                s = seq_shape(a, at.b);
            }
            const int64_t row = x / a.Hq;
            const int h = x % a.Hq, i = (int)row - a.cu[at.b], r = i * a.rep + h % a.rep;
            const Pieces w = pieces_of(a, at, s, h / a.rep, r, tot.units);
            if (a.whole && w.n == 1) continue;
            if (!a.part_inside(w.first / a.RB, w.n) || !a.row_inside(row)) continue;  // alike for all who share a barrier
            const float2 all = merged_ml(a, w, lane);
            float o[kC];
#pragma unroll
            for (int k = 0; k < kC; ++k) o[k] = 0.f;
            for (int p0 = wide == 1 ? 0 : warp; p0 < w.n; p0 += 8 * wide) {
                float m[8], v[8][kC];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int p = p0 + u * wide;
                    const int64_t e = w.first + (int64_t)p * a.RB;
                    m[u] = p < w.n ? a.part_ml[e].x : -INFINITY;
#pragma unroll
                    for (int k = 0; k < kC; ++k) v[u][k] = p < w.n ? a.part_o[e * D + k * 32 + lane] : 0.f;
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const float f = m[u] == all.x ? 1.f : ex2(m[u] - all.x);
#pragma unroll
                    for (int k = 0; k < kC; ++k) o[k] = fmaf(f, v[u][k], o[k]);
                }
            }
            const float inv = all.x == -INFINITY && all.y == 0.f ? 0.f : 1.f / all.y;
            char* to = a.out + (row * a.Hq + h) * D * (int64_t)sizeof(T);
            if (wide == 1) {
#pragma unroll
                for (int k = 0; k < kC; ++k) Unit<T>::put(to + (k * 32 + lane) * sizeof(T), o[k] * inv);
            } else {
                __syncthreads();  // the row before is written
#pragma unroll
                for (int k = 0; k < kC; ++k) part[warp][k * 32 + lane] = o[k];
                __syncthreads();
                if (t < D) Unit<T>::put(to + t * sizeof(T), ((part[0][t] + part[1][t]) + (part[2][t] + part[3][t])) * inv);
            }
            if (lane == 0 && (wide == 1 || warp == 0)) {
                if (a.lse != nullptr)
                    a.lse[(int64_t)h * a.n_rows + row] = all.y == 0.f ? -INFINITY : fmaf(all.x, kLn2, logf(all.y));
                if (a.factor != nullptr) a.factor[row * a.Hq + h] = weight_factor(a, all, row);
            }
        }
        return;
    }
    if (lost) return;
    // every warp for itself: an equal part of the block's items
    const int it0 = share_begin(c, tot.items, G), part = share_begin(c + 1, tot.items, G) - it0;
    float2* f = ml[warp];
    for_items(a, at, it0 + share_begin(warp, part, kThreads / 32), it0 + share_begin(warp + 1, part, kThreads / 32),
              [&](const Place& at, const SeqShape& s, int g, int tile0, int tile1) {
        const int64_t row0 = a.cu[at.b];
        const int R = s.n * a.rep;
        __syncwarp();
        if (a.whole && pieces_of(a, at, s, g, 0, tot.units).n == 1) {  // (kept scores of bf16: one block of rows)
            for (int r = lane; r < R; r += 32)
                f[r] = a.row_inside(row0 + r / a.rep) ? a.factor[(row0 + r / a.rep) * a.Hq + g * a.rep + r % a.rep] : make_float2(0.f, 0.f);
        } else {
            for (int rw = 0; rw < R; rw += 4) {  // 8 lanes a row
                const int r = rw + (lane >> 3);
                float M = -INFINITY, L = 0.f;
                if (r < R) {
                    Pieces w = pieces_of(a, at, s, g, r, tot.units);
                    if (!a.part_inside(w.first / a.RB, w.n)) w.n = 0;
                    for (int p0 = lane & 7; p0 < w.n; p0 += 32) {  // 4 in flight
                        float2 x[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            x[u] = p0 + 8 * u < w.n ? a.part_ml[w.first + (int64_t)(p0 + 8 * u) * a.RB] : make_float2(-INFINITY, 0.f);
#pragma unroll
                        for (int u = 0; u < 4; ++u) merge_ml(M, L, x[u]);
                    }
                }
                for (int o = 4; o > 0; o >>= 1)
                    merge_ml(M, L, make_float2(__shfl_xor_sync(0xffffffffu, M, o), __shfl_xor_sync(0xffffffffu, L, o)));
                if (r < R && (lane & 7) == 0) f[r] = weight_factor(a, make_float2(M, L), row0 + r / a.rep);
            }
        }
        __syncwarp();
        for (int tile = tile0; tile < tile1; ++tile) {
            const bool drafts = tile == s.nt - 1;
            const int slot = tile * kCacheTile + lane * 4;
            const int n = (drafts ? (a.kn != nullptr && a.w_new != nullptr ? s.n : 0)
                                  : (a.accumulate ? s.len - tile * kCacheTile : 0)) - lane * 4;
            if (n <= 0) continue;
            float* to = nullptr;
            float4 had = make_float4(0.f, 0.f, 0.f, 0.f), sum = had;
            if (!drafts) {  // 4 slots of one page
                const int64_t page = a.c.page_of(at.b, slot, a.status);
                if (page < 0 || !a.c.inside(page, slot, g, a.status)) continue;
                to = a.c.weight + a.c.meta(page, slot, g);
                if (n >= 4) had = *reinterpret_cast<const float4*>(to);
            }
            auto one = [&](float x, float2 y, float& s1) {
                if (x != -INFINITY) s1 = fmaf(ex2(fmaf(x, a.scale_log2, y.x)), y.y, s1);
            };
            for (int k = 0; k < s.nrb; ++k) {
                const int r0 = k * a.RB, nr = min(a.RB, R - r0);
                const int u = at.unit0 + (g * s.nrb + k) * s.nt + tile;
                if (!a.unit_inside(u)) break;
                const float4* z = reinterpret_cast<const float4*>(a.score + (int64_t)u * a.RB * kCacheTile) + lane;
                constexpr int kBatch = 4;  // rows in flight; 8 spill, 25 us more over 256 sequences of some 2k
                for (int q0 = 0; q0 < nr; q0 += kBatch) {
                    float4 x[kBatch];
#pragma unroll
                    for (int r = 0; r < kBatch; ++r)
                        if (q0 + r < nr) x[r] = z[(q0 + r) * (kCacheTile / 4)];
#pragma unroll
                    for (int r = 0; r < kBatch; ++r) {
                        const float2 y = q0 + r < nr ? f[r0 + q0 + r] : make_float2(0.f, 0.f);
                        if (y.y == 0.f) continue;
                        one(x[r].x, y, sum.x);
                        one(x[r].y, y, sum.y);
                        one(x[r].z, y, sum.z);
                        one(x[r].w, y, sum.w);
                    }
                }
            }
            if (drafts) {
                if (!a.row_inside(row0 + lane * 4, min(n, 4))) continue;
                float* d = a.w_new + (row0 + lane * 4) * a.c.Hkv + g;
                d[0] = sum.x;
                if (n > 1) d[a.c.Hkv] = sum.y;
                if (n > 2) d[2 * a.c.Hkv] = sum.z;
                if (n > 3) d[3 * a.c.Hkv] = sum.w;
            } else if (n >= 4) {
                *reinterpret_cast<float4*>(to) = make_float4(had.x + sum.x, had.y + sum.y, had.z + sum.z, had.w + sum.w);
            } else {
                to[0] += sum.x;
                if (n > 1) to[1] += sum.y;
                if (n > 2) to[2] += sum.z;
            }
        }
    });
}

// The weights with the scores formed again, fp32: a thread a key, the rows in blocks of kRows.
template <class T, int D>
__global__ void __launch_bounds__(kThreads, kBlocks) cache_weight_kernel(const CacheAttnArgs a) {
    __shared__ PlanScratch sc;
    __shared__ __align__(16) float q[kRows][D];
    __shared__ __align__(16) float zs[kThreads][kRows];
    __shared__ float2 ml[kRows];
    const int t = threadIdx.x;
    const int c = blockIdx.x, G = gridDim.x;
    Place at;
    const PlanTotals tot = plan(a, &sc, &at, [&](const Place& x, const SeqShape& s, const PlanTotals& all) {
        const int it = share_begin(c, all.items, G);
        return it >= x.item0 && it < x.item0 + s.items(a.c.Hkv);
    });
    await_stream();  // the factors are complete
    admit_next();
    if (!tot.ok || *a.timed_out != 0) return;
    for_items(a, at, share_begin(c, tot.items, G), share_begin(c + 1, tot.items, G),
              [&](const Place& at, const SeqShape& s, int g, int tile0, int tile1) {
        const int64_t row0 = a.cu[at.b];
        const int R = s.n * a.rep;
        for (int tile = tile0; tile < tile1; ++tile) {
            const bool drafts = tile == s.nt - 1;
            if (drafts ? a.w_new == nullptr : !a.accumulate) continue;
            const KeyRow kr = key_row(a, s, at.b, g, tile, t, D * (int)sizeof(T));
            float sum = 0.f;
            for (int r0 = 0; r0 < R; r0 += kRows) {
                const int nr = min(kRows, R - r0);
                __syncthreads();
                load_q<T, D>(a, q, at.b, g, r0, nr);
                if (t < nr) {
                    const int64_t row = row0 + (r0 + t) / a.rep;
                    ml[t] = a.row_inside(row) ? a.factor[row * a.Hq + g * a.rep + (r0 + t) % a.rep] : make_float2(0.f, 0.f);
                }
                __syncthreads();
                float z[kRows];
                dots<D>(q, kr.k, zs + (t & ~31), z);
                if (kr.k == nullptr) continue;
                const uint64_t seen = drafts ? rows_that_see(a, row0, s.n, t, r0, nr) : ~0ull;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (r >= nr || !(seen >> r & 1)) continue;
                    const float2 f = ml[r];
                    if (f.y != 0.f) sum = fmaf(ex2(fmaf(z[r], a.scale_log2, f.x)), f.y, sum);
                }
            }
            if (kr.k == nullptr) continue;
            if (drafts) {
                if (a.row_inside(row0 + t)) a.w_new[(row0 + t) * a.c.Hkv + g] = sum;
            } else if (in_bounds(kr.meta >= 0 && kr.meta < a.c.meta(a.c.n_pages, 0, 0), a.status)) {
                a.c.weight[kr.meta] += sum;
            }
        }
    });
}

template <class T, int D>
estp_status launch(estp_ctx* ctx, CacheAttnArgs& a, cudaStream_t st) {
    constexpr bool kTc = sizeof(T) == 2;
    a.RB = kRows;
    if (kTc) {
        const int rows = a.max_rows * a.rep;
        a.RB = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 128 ? 128 : 256;
    }
    a.whole = kTc;
    a.G = ctx->num_sms * (kTc ? 1 : kBlocks);
    const int64_t groups = (int64_t)a.c.Hkv * (a.n_rows * a.rep / a.RB + a.B);
    const int64_t slots = a.G + groups;
    // scores of every unit: at most n_slots / 128 + 2 B tiles a KV head, times the row blocks of the
    // largest sequence
    const int64_t nrb = ((int64_t)a.max_rows * a.rep + a.RB - 1) / a.RB;
    const int64_t units = (int64_t)a.c.Hkv * nrb * (a.n_slots / kCacheTile + 2 * (int64_t)a.B);
    a.n_parts = slots;
    a.n_units = units;
    if (2 * units > INT32_MAX || a.n_rows * a.Hq > INT32_MAX)
        return fail(ESTP_ERR_UNSUPPORTED, "max_slots and rows: more than 2^31 tiles of work, or rows times heads");
    const size_t o_bytes = align_up(sizeof(float) * (size_t)slots * a.RB * D, 256);
    const size_t ml_bytes = align_up(sizeof(float2) * (size_t)slots * a.RB, 256);
    const size_t z_bytes = sizeof(float) * (size_t)units * a.RB * kCacheTile;
    const bool weights = a.accumulate || a.w_new != nullptr;
    // Kept scores cost 8 bytes a row and key (a write and a read), forming them again a read of K
    // (D * sizeof(T) bytes a key): kept up to the break-even, and up to 2 GB of them.
    const int64_t R = (int64_t)a.max_rows * a.rep;
    a.store = weights && R <= kCacheMaxStored && R * 8 <= (int64_t)(D * sizeof(T)) && z_bytes <= (size_t(2) << 30);
    const bool again = weights && !a.store;
    const size_t f_bytes = weights ? align_up(sizeof(float2) * (size_t)(a.n_rows * a.Hq), 256) : 0;
    const size_t more = f_bytes + (a.store ? z_bytes : 0);
    estp_status s = ws_reserve(ctx, o_bytes + ml_bytes + more);
    if (s != ESTP_OK) return s;
    char* ws = static_cast<char*>(ctx->ws);
    a.part_o = reinterpret_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(ws + o_bytes);
    a.factor = weights ? reinterpret_cast<float2*>(ws + o_bytes + ml_bytes) : nullptr;
    a.score = a.store ? reinterpret_cast<float*>(ws + o_bytes + ml_bytes + f_bytes) : nullptr;
    cudaError_t e;
    if constexpr (kTc) {
        s = a.RB <= 32 ? launch_cache_fwd_tc(ctx, a, st) : launch_cache_rows_tc(ctx, a, st);
        if (s != ESTP_OK) return s;
    } else {
        e = launch_dependent(cache_fwd_kernel<T, D>, a.G, kThreads, 0, st, a);
        if (e != cudaSuccess) return cuda_fail(e, "cache attention launch");
    }
    // Few rows have many partials each (28 rows of one 32K sequence with 76: 17 us for a warp a row, 4 for
    // a block); many rows keep the GPU busy a warp each (6600 rows: 14 us, 30 for a block).  One wave of 8
    // blocks an SM: 2 for them and 6 for the items of kept scores, or all for them.
    const int64_t some = (a.store ? 2 : 8) * ctx->num_sms;
    a.row_warps = a.n_rows * a.Hq <= 2 * ctx->num_sms ? kThreads / 32 : 1;
    const int64_t row_blocks = (a.n_rows * a.Hq * a.row_warps + kThreads / 32 - 1) / (kThreads / 32);
    a.row_blocks = (int)(row_blocks < some ? row_blocks : some);
    const int64_t items = (int64_t)a.c.Hkv * (a.n_slots / kCacheTile + 2 * (int64_t)a.B), many = 6 * ctx->num_sms;
    const int item_blocks = a.store ? (int)(items < many ? items : many) : 0;
    e = launch_dependent(cache_finish_kernel<T, D>, a.row_blocks + item_blocks, kThreads, 0, st, a);
    if (e != cudaSuccess) return cuda_fail(e, "cache attention finish launch");
    if (!again) return ESTP_OK;
    if constexpr (kTc) {
        return launch_cache_weight_tc(ctx, a, st);
    } else {
        e = launch_dependent(cache_weight_kernel<T, D>, ctx->num_sms * kBlocks, kThreads, 0, st, a);
        return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache weight launch");
    }
}

}  // namespace

estp_status launch_cache_attention(estp_ctx* ctx, CacheAttnArgs& a, estp_dtype dtype, cudaStream_t st) {
    if (dtype == ESTP_BF16)
        return a.c.d == 128 ? launch<__nv_bfloat16, 128>(ctx, a, st) : launch<__nv_bfloat16, 64>(ctx, a, st);
    return a.c.d == 128 ? launch<float, 128>(ctx, a, st) : launch<float, 64>(ctx, a, st);
}

}  // namespace estp
