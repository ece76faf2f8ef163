// The forward half of the cache attention (see cache_attn.cu) for bf16 caches, on the tensor cores, for
// up to 32 rows a (sequence, KV head): single tokens and small draft trees.
//
// Such a call has few rows and many keys, so the keys take the 128 lanes of an MMA and the rows its
// columns: per tile of 128 keys and block of RB rows
//   S^T = K Q^T          M = 128 keys, N = RB (16 at least), K = D
//   P   = 2^(S^T c - m)  a thread a key; each P is split into two bf16 terms, P = hi + lo, so that
//                        the second product keeps 16 bits of it
//   O^T += V^T [hi lo]   M = D, N = 2 RB (hi and lo columns, added at the end), K = 128 keys
// V^T is the V tile as it is stored (MN-major A), P goes to shared memory with a thread's columns
// contiguous (MN-major B): nothing is transposed.  A head size of 64 fills M = 128 by reading V
// twice (a leading offset of 0).
//
// The running maximum m of a row only moves when a tile exceeds it by 2^8: a thread forms
// S c - m, the group votes on whether any is above 8, and only then are the tile's maxima reduced
// over the lanes and O and l rescaled.  P stays below 2^8, and m is an exact part of the result
// (every partial is relative to it).
//
// One persistent CTA per SM over the units of cache.cuh.
//   warps 0, 3 TMA producers of the K and of the V tiles, a ring each, a box a page (a lane each); warp
//              3 also loads the rows' Q, a segment ahead
//   warp 1     issues S, as far ahead as K tiles and S buffers allow
//   warp 2     issues O, as soon as a P is written
//   warps 4-11 two epilogue groups of 4 warps, each with its S (double-buffered) and O in tensor
//              memory and its P, which take the tiles in turn
// Apart they matter: one warp that issued both products, one that loaded both tiles and a table look-up
// a tile each cost up to 1 us a tile (256 rollouts: 512 us with them, 386 without).
//
// Keys past a sequence's slots hold anything: S^T has them replaced, their P is 0 and their V rows
// (up to the MMA's 16-key step) are zeroed in shared memory before the product, as 0 x NaN is not 0.
// A draft whose V is not finite is zeroed there too and added by itself to the rows that see it.
//
// Bound by the K and V bytes (64 KB of a tile take 1.45 us an SM at the copy rate; an epilogue group has
// two tiles' time for one): 256 sequences of some 2000 slots, 8 KV heads, 380 us where the bytes take 343.
// With short sequences by the turns between segments (2 to 4 us: the last tile's V check, the join, the walk), whose
// code has left the instruction caches each time, so it is kept short.  Every wait is bounded; on expiry the CTA records ESTP_ERR_TIMEOUT, the
// groups vote to leave, and copies and MMAs are drained before TMEM is freed.
#include "cache_tc.cuh"

namespace estp {
namespace {

// Two epilogue groups: they take the tiles of a segment in turn, each with a softmax of its own over the
// block's RB rows, joined at its end.
constexpr int kGroups = 2;

template <int D, int RB>
struct Shape {
    static constexpr int kN = RB < 16 ? 16 : RB;  // S columns: an MMA of M = 128 has N >= 16
    static constexpr int kAtoms = D / 64;
    static constexpr int kTileBytes = kAtoms * kAtom;
    static constexpr int kQBufs = 2;              // the next segment's Q loads ahead
    static constexpr int kRowArrays = 5;          // [RB] floats a group keeps
    static constexpr int kQBytes = kAtoms * kN * 128;
    // P: [128 keys] rows of 128 bytes, hi then lo; of up to 16 rows both groups' P share one
    static constexpr int kPStep = RB == 32 ? kAtom : 64;  // from a group's P to the other's
    static constexpr int kPBytes = RB == 32 ? 2 * kAtom : kAtom;
    static constexpr int kFixed = kQBufs * kQBytes + kPBytes;
    static constexpr int kRoom = 227 * 1024 - 1024 - kFixed - 400 - kGroups * (kRowArrays + 4) * RB * 4;
    static constexpr int kStages = kRoom / kTileBytes < 12 ? kRoom / kTileBytes : 12;
    static constexpr int kKStages = (kStages - 1) / 2;  // a V tile waits through the softmax: 3 + 3 slots cost 16 of 445 us, 4 + 2 30
    static constexpr int kThreads = 128 + 128 * kGroups;
    static constexpr int kTmemUsed = kGroups * (2 * kN + 2 * RB);  // S twice, O hi and lo
    static constexpr int kTmem = kTmemUsed <= 128 ? 128 : kTmemUsed <= 256 ? 256 : 512;
    static constexpr int kOCol = kGroups * 2 * kN;
    // offsets from a 1024-aligned base
    static constexpr int kPOff = kStages * kTileBytes;
    static constexpr int kQOff = kPOff + kPBytes;
    static constexpr int kRedOff = kQOff + kQBufs * kQBytes;   // a group's [4][RB] per-warp values
    static constexpr int kBarOff = kRedOff + kGroups * 4 * RB * 4;
    static constexpr int kBars = 2 * kStages + 2 * kQBufs + 6 * kGroups + 2;
    static constexpr int kMiscOff = kBarOff + (kBars * 8 + 15) / 16 * 16;  // tmem address, abort flag, tiles issued, odd drafts
    static constexpr int kRowOff = kMiscOff + 48;  // a group's row arrays
    static constexpr int kSmem = kRowOff + kGroups * kRowArrays * RB * 4 + 1024;
    static_assert(kStages >= 4 && kSmem <= 227 * 1024, "shared memory per CTA");
};

// Reduces N columns (8, 16 or 32) over the warp's lanes; lane k returns with column k % N.  Every step
// halves the columns a lane still holds.
template <int N, class Op>
__device__ __forceinline__ float reduce_scatter(const float* z, int lane, Op op) {
    float v[N / 2];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        const bool up = lane & (N / 2);
        v[k] = op(up ? z[k + N / 2] : z[k], __shfl_xor_sync(0xffffffffu, up ? z[k] : z[k + N / 2], N / 2));
    }
#pragma unroll
    for (int o = N / 4; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < o; ++k) {
            const bool up = lane & o;
            v[k] = op(up ? v[k + o] : v[k], __shfl_xor_sync(0xffffffffu, up ? v[k] : v[k + o], o));
        }
#pragma unroll
    for (int o = N; o < 32; o <<= 1) v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], o));
    return v[0];
}

template <int D, int RB>
__global__ void __launch_bounds__(Shape<D, RB>::kThreads, 1)
    cache_fwd_tc_kernel(const __grid_constant__ TcMaps tm, const CacheAttnArgs a, const int box_rows, const int new_rows) {
    using S = Shape<D, RB>;
    constexpr int NB = kGroups;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + S::kBarOff);  // [kStages], K then V
    uint64_t* empty = full + S::kStages;                            // [kStages]
    const Ring ring_k{full, empty, sm, S::kKStages, S::kTileBytes};
    const Ring ring_v{full + S::kKStages, empty + S::kKStages, sm + S::kKStages * S::kTileBytes, S::kStages - S::kKStages, S::kTileBytes};
    uint64_t* q_full = empty + S::kStages;                          // [kQBufs]
    uint64_t* q_empty = q_full + S::kQBufs;                         // [kQBufs]
    uint64_t* s_full = q_empty + S::kQBufs;                         // [NB][2]
    uint64_t* s_empty = s_full + 2 * NB;                            // [NB][2]
    uint64_t* p_full = s_empty + 2 * NB;                            // [NB]
    uint64_t* pv_done = p_full + NB;                                // [NB]
    uint64_t* drain = pv_done + NB;                                 // [2] each issuer's MMAs done
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + S::kMiscOff);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::kMiscOff + 4);
    volatile int* issued_tiles = reinterpret_cast<volatile int*>(sm + S::kMiscOff + 8);  // [2] K, V
    volatile uint32_t* odd = reinterpret_cast<volatile uint32_t*>(sm + S::kMiscOff + 16);  // [2][4] drafts with V not finite

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < S::kQBufs; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < NB; ++i) {
            mbar_init(&s_full[2 * i], 1);
            mbar_init(&s_full[2 * i + 1], 1);
            mbar_init(&s_empty[2 * i], 4);
            mbar_init(&s_empty[2 * i + 1], 4);
            mbar_init(&p_full[i], 4);
            mbar_init(&pv_done[i], 1);
        }
        mbar_init(&drain[0], 1);
        mbar_init(&drain[1], 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(S::kTmem));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    await_stream();
    const int cta = blockIdx.x;
    // the plan's scratch lies in the ring, which is unused until the barrier below
    Walk walk{Place{0, 0, 0, 0}, 0, 0};
    Place place;
    const PlanTotals tot = plan(a, reinterpret_cast<PlanScratch*>(sm), &place, [&](const Place& x, const SeqShape& s, const PlanTotals& all) {
        const int u = share_begin(cta, all.units, ctas_of(a, all.units));
        return u >= x.unit0 && u < x.unit0 + s.units(a.c.Hkv);
    });
    const uint32_t tmem = *tmem_slot;
    const int G = ctas_of(a, tot.units);
    if (tot.ok && cta < G) walk = Walk{place, share_begin(cta, tot.units, G), share_begin(cta + 1, tot.units, G)};
    if (a.B > 32) {  // the plan used its scratch
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    Segment sg;

    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------ producers
        // warp 0 the K tiles, warp 3 the V tiles and the rows' Q
        const int kv = warp == 3;
        const Ring ring = kv ? ring_v : ring_k;
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(
                          kv ? (lane ? &tm.vn : &tm.v) : (lane ? &tm.kn : &tm.k))) : "memory");
        uint32_t t = 0, q_seg = 0;  // tiles issued; segments whose Q is loaded
        bool ok = true;
        Walk q_walk = walk;
        Segment qs;
        // Q of the next segment (zeros past its rows), K-major with the 128-byte swizzle
        auto load_q = [&]() {
            if (!q_walk.next<RB>(a, qs)) return;
            const uint32_t qb = q_seg % S::kQBufs, use = q_seg / S::kQBufs;
            if (use >= 1 && !warp_wait(&q_empty[qb], (use - 1) & 1, abort_flag, a.status, a.wait_cycles)) {
                ok = false;
                return;
            }
            ++q_seg;
            const int64_t row0 = a.cu[qs.b];
            const uint32_t to = smem_u32(sm + S::kQOff + qb * S::kQBytes);
            constexpr int kTogether = 32 / (D / 8);  // rows at a time
            const int ch = lane % (D / 8);
            int i = (qs.r0 + lane / (D / 8)) / a.rep, h = (qs.r0 + lane / (D / 8)) % a.rep;
#pragma unroll 1
            for (int r = lane / (D / 8); r < S::kN; r += kTogether) {
                const char* from = a.Q + ch * 16;
                if (r < qs.nr) from += (row0 + i) * a.ldq + (int64_t)(qs.g * a.rep + h) * (D * 2);
                for (h += kTogether; h >= a.rep; h -= a.rep) ++i;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                 to + (ch >> 3) * S::kN * 128 + r * 128 + (((ch & 7) ^ (r & 7)) << 4)),
                             "l"(from), "r"(r < qs.nr ? 16 : 0)
                             : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full[qb]);
        };
        if (kv) load_q();
        PageWindow win;
        while (ok && walk.next<RB>(a, sg)) {
            win.open(a, sg.s, sg.b, sg.tile0, lane);
            for (int tile = sg.tile0; tile < sg.tile1; ++tile, ++t) {
                if (t >= (uint32_t)ring.n && !warp_wait(ring.freed(t), ring.parity(t - ring.n), abort_flag, a.status, a.wait_cycles)) {
                    ok = false;
                    break;
                }
                load_tile<D>(a, kv ? &tm.v : &tm.k, kv ? &tm.vn : &tm.kn, win, sg.s, sg.b, sg.g, tile, box_rows, new_rows,
                             ring.tile(t), ring.filled(t), lane);
                if (kv && tile == sg.tile0) load_q();  // a failure shows at the next wait
            }
        }
        if (lane == 0) issued_tiles[kv] = (int)t;
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ S issuer
        if (lane == 0) {
            constexpr uint32_t kIdS = idesc_bf16(kCacheTile, S::kN);
            uint32_t t = 0, seg = 0;   // tiles and segments begun
            uint32_t steps[NB] = {};   // S issued for a group
            bool ok = true, issued = false;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = ok && wait_bar(bar, parity, abort_flag, a.status, a.wait_cycles);
                return ok;
            };
            while (ok && walk.next<RB>(a, sg)) {
                const int tiles = sg.tile1 - sg.tile0;
                const uint32_t qb = seg % S::kQBufs;
                if (!wait(&q_full[qb], (seg / S::kQBufs) & 1)) break;
                ++seg;
                for (int i = 0; ok && i < tiles; ++i, ++t) {
                    if (!wait(ring_k.filled(t), ring_k.parity(t))) break;
                    const uint32_t ka = smem_u32(ring_k.tile(t));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        if ((i & 1) != nb) continue;
                        const uint32_t n = steps[nb]++, buf = n & 1, use = n >> 1;
                        if (use >= 1 && !wait(&s_empty[2 * nb + buf], (use - 1) & 1)) break;
                        tc_fence_after();
                        issued = true;
                        product_k_major<kIdS, D>(tmem + (2 * nb + buf) * S::kN, ka, kAtom,
                                                 smem_u32(sm + S::kQOff + qb * S::kQBytes), S::kN * 128);
                        mma_commit(&s_full[2 * nb + buf]);
                    }
                    if (ok) mma_commit(ring_k.freed(t));
                }
                if (ok) mma_commit(&q_empty[qb]);
            }
            if (issued) {
                mma_commit(&drain[0]);
                drain_wait(&drain[0], 0, a.status);
            }
        }
        __syncwarp();
    } else if (warp == 2) {
        // ------------------------------------------------------------ O issuer
        // apart from S, whose wait for the next K must not hold back a finished P and the V slot behind it
        if (lane == 0) {
            constexpr uint32_t kIdO = idesc_bf16(kCacheTile, 2 * RB) | (1u << 15) | (1u << 16);  // both MN-major
            uint32_t t = 0, pv[NB] = {};
            bool ok = true, issued = false;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = ok && wait_bar(bar, parity, abort_flag, a.status, a.wait_cycles);
                return ok;
            };
            while (ok && walk.next<RB>(a, sg)) {
                const int tiles = sg.tile1 - sg.tile0;
                bool live[NB] = {};  // a group's O holds a product of this segment
                for (int i = 0; ok && i < tiles; ++i, ++t) {
                    if (!wait(ring_v.filled(t), ring_v.parity(t))) break;
                    const uint32_t va = smem_u32(ring_v.tile(t));
                    const int ksteps = (tile_keys(a, sg.s, sg.tile0 + i) + 15) / 16;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        if ((i & 1) != nb) continue;
                        if (!wait(&p_full[nb], pv[nb]++ & 1)) break;
                        tc_fence_after();
                        issued = true;
                        const uint32_t pa = smem_u32(sm + S::kPOff) + nb * S::kPStep;
                        for (int kk = 0; kk < ksteps; ++kk)
                            mma_bf16<kIdO>(tmem + (uint32_t)(S::kOCol + nb * 2 * RB), mn_desc(va + kk * 2048, D == 128 ? kAtom : 0),
                                           mn_desc(pa + kk * 2048, kAtom), live[nb] || kk > 0 ? 1u : 0u);
                        mma_commit(&pv_done[nb]);
                        live[nb] = live[nb] || ksteps > 0;
                    }
                    if (ok) mma_commit(ring_v.freed(t));
                }
            }
            if (issued) {
                mma_commit(&drain[1]);
                drain_wait(&drain[1], 0, a.status);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------- epilogue
        const int nb = (warp - 4) >> 2, q = warp & 3, bar = 1 + nb;
        const int j = q * 32 + lane;                 // key of the tile; lane of S and O
        float* row_m = reinterpret_cast<float*>(sm + S::kRowOff) + nb * S::kRowArrays * RB;  // m, log2 units
        float* row_f = row_m + RB;                   // rescaling factors; l at the end of a segment
        float* row_n = row_f + RB;                   // -m, or 0 where m is -inf
        uint8_t* pb = sm + S::kPOff;
        float* row_w = reinterpret_cast<float*>(sm + S::kRedOff) + nb * 4 * RB;  // [4][RB]
        volatile uint32_t* odd_drafts = odd + nb * 4;
        // 16-byte chunk c of key k's P row of a group
        auto p_chunk = [&](int group, int k, int c) {
            if (RB == 32) return pb + group * S::kPStep + k * 128 + ((c ^ (k & 7)) << 4);
            return pb + k * 128 + (((group * (S::kPStep / 16) + c) ^ (k & 7)) << 4);
        };
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t t_o = tmem + lane_off + (uint32_t)(S::kOCol + nb * 2 * RB);
        constexpr int kCols = RB < 16 ? 8 : 16;  // columns of a tensor memory load
        uint32_t step = 0, t = 0;
        bool alive = true;
        auto wait = [&](uint64_t* b, uint32_t parity) {
            if (alive) alive = warp_wait(b, parity, abort_flag, a.status, a.wait_cycles);
        };
        while (walk.next<RB>(a, sg)) {
            const int nr = sg.nr;
            const int64_t row0 = a.cu[sg.b];
            if (j < RB) row_m[j] = -INFINITY;
            float2 l[RB / 2];
#pragma unroll
            for (int r = 0; r < RB / 2; ++r) l[r] = make_float2(0.f, 0.f);
            bool live = false, lost = true;  // lost: a row has no m yet, every tile looks for one
            const int first = sg.tile0 + nb;
            const float2 c2 = make_float2(a.scale_log2, a.scale_log2);
            for (int tile = first; tile < sg.tile1; tile += kGroups, ++step) {
                const bool drafts = tile == sg.s.nt - 1;
                const int keys = tile_keys(a, sg.s, tile);
                const uint32_t buf = step & 1;
                uint64_t seen = ~0ull;  // rows that see this thread's key
                if (drafts) seen = rows_that_see(a, row0, keys, j, sg.r0, nr);
                else if (j >= keys) seen = 0;
                wait(&s_full[2 * nb + buf], (step >> 1) & 1);
                tc_fence_after();
                float z[RB];
                auto load_s = [&]() {
#pragma unroll
                    for (int r = 0; r < RB; r += kCols)
                        tmem_ld_cols<kCols>(tmem + lane_off + (2 * nb + buf) * S::kN + r, z + r);
                    tmem_wait_ld();
                    tie<RB>(z);
                    if (drafts || keys < kCacheTile) {
#pragma unroll
                        for (int r = 0; r < RB; ++r)
                            if (!(seen >> r & 1)) z[r] = -INFINITY;
                    }
                };
                load_s();
                if (a.store && alive && a.unit_inside(walk.u - (sg.tile1 - tile))) {
                    float* to = a.score + ((int64_t)(walk.u - (sg.tile1 - tile)) * a.RB) * kCacheTile + j;
#pragma unroll
                    for (int r = 0; r < RB; ++r)
                        if (r < nr) to[r * kCacheTile] = z[r];
                }
                // S c - m; does any score exceed its row's m by 2^8?
                float top = -INFINITY;
                auto relative = [&]() {
#pragma unroll
                    for (int r = 0; r < RB; r += 4) {
                        const float4 n = *reinterpret_cast<const float4*>(row_n + r);
                        const float2 x = __ffma2_rn(make_float2(z[r], z[r + 1]), c2, make_float2(n.x, n.y));
                        const float2 y = __ffma2_rn(make_float2(z[r + 2], z[r + 3]), c2, make_float2(n.z, n.w));
                        z[r] = x.x;
                        z[r + 1] = x.y;
                        z[r + 2] = y.x;
                        z[r + 3] = y.y;
                        top = fmax3(fmax3(top, x.x, x.y), y.x, y.y);
                    }
                };
                if (!lost) relative();
                if (group_or(bar, lost || top > 8.f || !alive)) {
                    if (step > 0) wait(&pv_done[nb], (step - 1) & 1);
                    tc_fence_after();
                    if (group_or(bar, !alive)) {
                        alive = false;
                        break;
                    }
                    if (!lost) load_s();
                    const float x = reduce_scatter<RB>(z, lane, [](float a, float b) { return fmaxf(a, b); });
                    if (lane < RB) row_w[q * RB + lane] = x;
                    group_sync(bar);
                    bool none = false;
                    if (j < RB) {
                        const float x = fmaxf(fmaxf(row_w[j], row_w[RB + j]), fmaxf(row_w[2 * RB + j], row_w[3 * RB + j]));
                        const float old = row_m[j], m = fmaxf(old, x * a.scale_log2);
                        none = m == -INFINITY;
                        row_f[j] = old == m ? 1.f : ex2(old - m);
                        row_m[j] = m;
                        row_n[j] = none ? 0.f : -m;
                    }
                    lost = group_or(bar, none);
#pragma unroll
                    for (int r = 0; r < RB; r += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(row_f + r);
                        l[r / 2] = __fmul2_rn(l[r / 2], make_float2(f.x, f.y));
                        l[r / 2 + 1] = __fmul2_rn(l[r / 2 + 1], make_float2(f.z, f.w));
                    }
                    if (live) {
#pragma unroll 1
                        for (int c = 0; c < 2 * RB; c += 16) {
                            float o[16];
                            tmem_ld16(t_o + c, o);
                            tmem_wait_ld();
                            tie<16>(o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] *= row_f[(c + k) % RB];
                            tmem_st16(t_o + c, o);
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    }
                    relative();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&s_empty[2 * nb + buf]);
                // P in place of the scores
#pragma unroll
                for (int r = 0; r < RB; r += 2) {
                    z[r] = ex2(z[r]);
                    z[r + 1] = ex2(z[r + 1]);
                    l[r / 2] = __fadd2_rn(l[r / 2], make_float2(z[r], z[r + 1]));
                }
                if (step > 0) wait(&pv_done[nb], (step - 1) & 1);  // the P buffer is free
#pragma unroll
                for (int r = 0; r < RB; r += 8) {
                    uint4 h, lo;
                    h.x = pack_hi_lo(z[r], z[r + 1], lo.x);
                    h.y = pack_hi_lo(z[r + 2], z[r + 3], lo.y);
                    h.z = pack_hi_lo(z[r + 4], z[r + 5], lo.z);
                    h.w = pack_hi_lo(z[r + 6], z[r + 7], lo.w);
                    *reinterpret_cast<uint4*>(p_chunk(nb, j, r / 8)) = h;
                    *reinterpret_cast<uint4*>(p_chunk(nb, j, (r + RB) / 8)) = lo;
                }
                if (drafts || (keys & 15)) {
                    // V rows that must not reach the product: past the keys, and drafts that are not finite
                    const uint32_t tv = t + (tile - sg.tile0);
                    wait(ring_v.filled(tv), ring_v.parity(tv));
                    uint8_t* vr = ring_v.tile(tv) + j * 128;
                    bool clear = j >= keys && j < ((keys + 15) & ~15);
                    if (drafts && j < keys) clear = row_not_finite<D>(vr);
                    if (drafts) {
                        const unsigned bits = __ballot_sync(0xffffffffu, clear && j < keys);
                        if (lane == 0) odd_drafts[q] = bits;
                    }
                    if (clear) clear_row<D>(vr);
                }
                tc_fence_before();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[nb]);
                live = live || keys > 0;
            }
            t += sg.tile1 - sg.tile0;
            // the segment's partial
            if (step > 0) wait(&pv_done[nb], (step - 1) & 1);
            // a segment that is its whole group is finished here, by both epilogue groups
            const bool whole = sg.tile0 == 0 && sg.tile1 == sg.s.nt;
            if (both_groups_or(!alive)) break;  // who shares barriers leaves together
            tc_fence_after();
            // drafts whose V is not finite were left out of O: their P is still in its buffer, row by row
            if (sg.tile1 == sg.s.nt && ((sg.tile1 - 1 - sg.tile0) & 1) == nb &&
                (odd_drafts[0] | odd_drafts[1] | odd_drafts[2] | odd_drafts[3])) {
#pragma unroll 1
                for (int r = 0; r < nr; ++r) {
                    float s = 0.f;
#pragma unroll 1
                    for (int x = 0; x < sg.s.n; ++x) {
                        if ((D == 64 && q >= 2) || !(odd_drafts[x >> 5] >> (x & 31) & 1)) continue;
                        if (!(rows_that_see(a, row0, sg.s.n, x, sg.r0 + r, 1) & 1)) continue;
                        const float v = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(
                            a.vn + (row0 + x) * a.ldn + (int64_t)sg.g * (D * 2) + j * 2));
                        const __nv_bfloat16* ph = reinterpret_cast<const __nv_bfloat16*>(p_chunk(nb, x, r >> 3)) + (r & 7);
                        const __nv_bfloat16* pl = reinterpret_cast<const __nv_bfloat16*>(p_chunk(nb, x, (r + RB) >> 3)) + (r & 7);
                        s += (__bfloat162float(*ph) + __bfloat162float(*pl)) * v;
                    }
                    __syncwarp();
                    uint32_t o;
                    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(o) : "r"(t_o + r));
                    tmem_wait_ld();
                    asm volatile("" : "+r"(o));
                    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(t_o + r),
                                 "r"(__float_as_uint(__uint_as_float(o) + s))
                                 : "memory");
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
            }
            // l over the keys' threads, into row_f
            {
                const auto plus = [](float x, float y) { return x + y; };
                float v[RB];
#pragma unroll
                for (int k = 0; k < RB; k += 2) {
                    v[k] = l[k / 2].x;
                    v[k + 1] = l[k / 2].y;
                }
                const float x = reduce_scatter<RB>(v, lane, plus);
                if (lane < RB) row_w[q * RB + lane] = x;
            }
            group_sync(bar);
            if (j < RB) row_f[j] = (row_w[j] + row_w[RB + j]) + (row_w[2 * RB + j] + row_w[3 * RB + j]);
            // the groups' halves joined: what their O count (a group without a key counts 0), and the whole's scale
            float* row_a = row_n + RB;
            float* row_b = row_a + RB;
            tc_fence_before();
            both_groups_or(false);
            tc_fence_after();
            const int64_t part = (int64_t)(cta + sg.group) * a.RB;
            if (j < RB) {
                const float *m0 = reinterpret_cast<const float*>(sm + S::kRowOff), *m1 = m0 + S::kRowArrays * RB;
                const float ma = m0[j], mb = m1[j], la = m0[RB + j], lb = m1[RB + j], M = fmaxf(ma, mb);
                float fa = ma == -INFINITY ? 0.f : ex2(ma - M), fb = mb == -INFINITY ? 0.f : ex2(mb - M);
                // a group without a maximum adds nothing, or NaN, which stays
                const float L = (fa != 0.f ? fa * la : M == -INFINITY ? la : 0.f) + (fb != 0.f ? fb * lb : M == -INFINITY ? lb : 0.f);
                if (L != L) fa = fb = 1.f;
                const float scale = !whole ? 1.f : M == -INFINITY && L == 0.f ? 0.f : 1.f / L;
                row_a[j] = fa * scale;
                row_b[j] = fb * scale;
                if (nb == 0 && j < nr && (whole ? a.row_inside(row0 + (sg.r0 + j) / a.rep) : a.part_inside(cta + sg.group))) {
                    if (whole) {
                        const int rr = sg.r0 + j, h = sg.g * a.rep + rr % a.rep;
                        const int64_t row = row0 + rr / a.rep;
                        if (a.lse != nullptr) a.lse[(int64_t)h * a.n_rows + row] = L == 0.f ? -INFINITY : fmaf(M, kLn2, logf(L));
                        if (a.factor != nullptr) a.factor[row * a.Hq + h] = weight_factor(a, make_float2(M, L), row);
                    } else {
                        a.part_ml[part + j] = make_float2(M, L);
                    }
                }
            }
            group_sync(bar);
            // O of half the rows a group: lane = column
            constexpr int kMine = RB / 2;
            const uint32_t t_a = tmem + lane_off + (uint32_t)S::kOCol;
            {
                const int r = nb * kMine;
                float hi[kMine], lo[kMine], hb[kMine], lb[kMine];
                tmem_ld_cols<kMine>(t_a + r, hi);
                tmem_ld_cols<kMine>(t_a + RB + r, lo);
                tmem_ld_cols<kMine>(t_a + 2 * RB + r, hb);
                tmem_ld_cols<kMine>(t_a + 3 * RB + r, lb);
                tmem_wait_ld();
                tie<kMine>(hi);
                tie<kMine>(lo);
                tie<kMine>(hb);
                tie<kMine>(lb);
                if (D == 128 || q < 2) {
                    int i = (sg.r0 + r) / a.rep, h = sg.g * a.rep + (sg.r0 + r) % a.rep;  // draft and head of the row
#pragma unroll
                    for (int k = 0; k < kMine; ++k) {
                        if (r + k >= nr) break;
                        const float wa = row_a[r + k], wb = row_b[r + k];
                        float o = wa != 0.f ? (hi[k] + lo[k]) * wa : 0.f;
                        if (wb != 0.f) o = fmaf(hb[k] + lb[k], wb, o);
                        if (whole) {
                            if (a.row_inside(row0 + i))
                                reinterpret_cast<__nv_bfloat16*>(a.out)[((row0 + i) * a.Hq + h) * D + j] = __float2bfloat16_rn(o);
                        } else if (a.part_inside(cta + sg.group)) {
                            a.part_o[(part + r + k) * D + j] = o;
                        }
                        if (++h == (sg.g + 1) * a.rep) ++i, h -= a.rep;
                    }
                }
            }
            tc_fence_before();
            both_groups_or(false);  // O is read: the next segment's may begin
            tc_fence_before();
            group_sync(bar);  // row_w, row_m and P are free for the next segment
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    admit_next();  // (earlier, the next kernel's waiting blocks cost this one 3 %)
    if (threadIdx.x == 0 && *abort_flag) {
        *a.timed_out = 1;  // the partials and scores are not all there
        ring_k.drain(issued_tiles[0], a.status);
        ring_v.drain(issued_tiles[1], a.status);
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmem));
    }
}

template <int D, int RB>
estp_status launch(estp_ctx* ctx, const TcMaps& tm, const CacheAttnArgs& a, int box_rows, int new_rows, cudaStream_t st) {
    using S = Shape<D, RB>;
    const int bit = 2 + (D == 128 ? 8 : 0) + (RB == 8 ? 0 : RB == 16 ? 1 : 2);
    cudaError_t e = set_smem(ctx, bit, cache_fwd_tc_kernel<D, RB>, S::kSmem);
    if (e != cudaSuccess) return cuda_fail(e, "cache attention smem attribute");
    e = launch_dependent(cache_fwd_tc_kernel<D, RB>, a.G, S::kThreads, S::kSmem, st, tm, a, box_rows, new_rows);
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache attention launch");
}

template <int D>
estp_status launch_rows(estp_ctx* ctx, const TcMaps& tm, const CacheAttnArgs& a, int box_rows, int new_rows, cudaStream_t st) {
    switch (a.RB) {
        case 8: return launch<D, 8>(ctx, tm, a, box_rows, new_rows, st);
        case 16: return launch<D, 16>(ctx, tm, a, box_rows, new_rows, st);
        default: return launch<D, 32>(ctx, tm, a, box_rows, new_rows, st);
    }
}

}  // namespace

estp_status launch_cache_fwd_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st) {
    TcMaps tm;
    int box_rows, new_rows;
    const estp_status s = make_maps(a, &tm, &box_rows, &new_rows);
    if (s != ESTP_OK) return s;
    return a.c.d == 128 ? launch_rows<128>(ctx, tm, a, box_rows, new_rows, st) : launch_rows<64>(ctx, tm, a, box_rows, new_rows, st);
}

}  // namespace estp
