// The cache attention's weights with the scores formed again (see cache_attn.cu) for bf16 caches:
// S^T = K Q^T tile by tile with every row of the (b, KV head) resident, 128 rows a product (64 take the
// tensor pipe as long), w_j = sum_r c_r 2^(S_jr c - M_r) / L_r, a thread a key.  A CTA takes an equal run
// of the call's (b, KV head, tile), which go to the two epilogue groups in turn, all rows of a tile to
// one.  Where 64 rows all count, two at a time in packed FMAs; else each by the mask of rows that see
// the key and have a factor (a factor of 0 must not meet a score that is not finite).  Rows beyond
// kWRows take another pass over the run, by the same threads.
// Bound by K's bytes up to some 170 rows a KV head (8 sequences of 8k: a tile each 0.84 us, 5.9 TB/s), then
// by ex2 and the issue of the sums.
#include "cache_tc.cuh"

namespace estp {
namespace {

constexpr int kWRows = 448, kWBlock = 64, kWMinStages = 3, kWMaxStages = 6, kWBufs = 2;
constexpr int kWCols = 2 * kWBlock;  // of one product: two blocks of rows, the last perhaps one
template <int D>
struct WShape {
    static constexpr int kAtoms = D / 64;
    static constexpr int kTileBytes = kAtoms * kAtom;
    static constexpr int kBlockBytes = kAtoms * kWBlock * 128;  // Q of one block of rows
    // from a 1024-aligned base: barriers, factors and sums first, then Q blocks and as many K tiles as fit
    static constexpr int kBars = 2 * kWMaxStages + 1 + 4 * kWBufs + 1;
    static constexpr int kMiscOff = kBars * 8;          // tmem address, abort flag
    static constexpr int kNzOff = kMiscOff + 16;        // [kWRows / 32] rows with a factor
    static constexpr int kFOff = 256;                   // [kWRows / 2][4] factors of two rows: offsets, then multiples
    static constexpr int kQOff = (kFOff + kWRows * 8 + 1023) / 1024 * 1024;
    static_assert(kNzOff + kWRows / 8 <= kFOff, "barriers");
    static constexpr int kThreads = 64 + 256;
    static constexpr int kRoom = 227 * 1024 - 1024 - kQOff;
    static int stages(int blocks) {
        const int n = (kRoom - blocks * kBlockBytes) / kTileBytes;
        return n < kWMaxStages ? n : kWMaxStages;
    }
    static int smem(int blocks) { return 1024 + kQOff + blocks * kBlockBytes + stages(blocks) * kTileBytes; }
    static_assert(kRoom - kWRows / kWBlock * kBlockBytes >= kWMinStages * kTileBytes, "shared memory per CTA");
};

// Runs of one (b, KV head) in items [it, it1).
struct ItemWalk {
    Place at;
    int it, it1;
    SeqShape s;
    int b, g, tile0, tile1;
    __device__ __forceinline__ bool next(const CacheAttnArgs& a) {
        while (it < it1) {
            s = seq_shape(a, at.b);
            if (it >= at.item0 + s.items(a.c.Hkv)) {
                at.pass(s, a.c.Hkv);
                continue;
            }
            b = at.b;
            g = (it - at.item0) / s.nt;
            tile0 = (it - at.item0) % s.nt;
            tile1 = min(s.nt, tile0 + (it1 - it));
            it += tile1 - tile0;
            // tiles whose weight no one asks for
            if (!a.accumulate) tile0 = max(tile0, s.nt - 1);
            if (a.w_new == nullptr) tile1 = min(tile1, s.nt - 1);
            if (tile0 < tile1) return true;
        }
        return false;
    }
};

template <int D>
__global__ void __launch_bounds__(WShape<D>::kThreads, 1)
    cache_weight_tc_kernel(const __grid_constant__ TcMaps tm, const CacheAttnArgs a, const int box_rows, const int new_rows,
                           const int q_blocks, const int n_stages) {
    using S = WShape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
    uint8_t* ring = sm + S::kQOff + q_blocks * S::kBlockBytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm);  // [kWMaxStages]
    uint64_t* empty = full + kWMaxStages;
    uint64_t* q_full = empty + kWMaxStages;
    uint64_t* s_full = q_full + 1;          // [2][kWBufs]
    uint64_t* s_empty = s_full + 2 * kWBufs;
    uint64_t* drain = s_empty + 2 * kWBufs;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + S::kMiscOff);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::kMiscOff + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWMaxStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(q_full, 8);
        for (int i = 0; i < 2 * kWBufs; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], 4);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(2 * kWBufs * kWCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int cta = blockIdx.x, G = gridDim.x;
    Place place;
    const PlanTotals tot = plan(a, reinterpret_cast<PlanScratch*>(ring), &place, [&](const Place& x, const SeqShape& s, const PlanTotals& all) {
        const int it = share_begin(cta, all.items, G);
        return it >= x.item0 && it < x.item0 + s.items(a.c.Hkv);
    });
    ItemWalk w{Place{0, 0, 0, 0}, 0, 0};
    if (tot.ok) {
        w.it = share_begin(cta, tot.items, G);
        w.it1 = share_begin(cta + 1, tot.items, G);
        w.at = place;
    }
    if (a.B > 32) {  // the plan used its scratch, in the ring
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    await_stream();  // the factors are complete
    admit_next();

    if (warp == 0) {
        // ------------------------------------------------------------ producer
        uint32_t e = 0;
        bool ok = true;
        PageWindow win;
        while (ok && w.next(a)) {
            for (int r0 = 0; ok && r0 < w.s.n * a.rep; r0 += kWRows) {
                win.open(a, w.s, w.b, w.tile0, lane);
                for (int tile = w.tile0; tile < w.tile1; ++tile, ++e) {
                    const int slot = (int)(e % n_stages);
                    const uint32_t use = e / n_stages;
                    if (use >= 1 && !warp_wait(&empty[slot], (use - 1) & 1, abort_flag, a.status, a.wait_cycles)) {
                        ok = false;
                        break;
                    }
                    load_tile<D>(a, &tm.k, &tm.kn, win, w.s, w.b, w.g, tile, box_rows, new_rows, ring + slot * S::kTileBytes,
                                 &full[slot], lane);
                }
            }
        }
        if (lane == 0)
            for (uint32_t i = 0; i < (uint32_t)n_stages && i < e; ++i)
                drain_wait(&full[(e - 1 - i) % n_stages], ((e - 1 - i) / n_stages) & 1, a.status);
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------- MMA issuer
        if (lane == 0) {
            constexpr uint32_t kId2 = idesc_bf16(kCacheTile, kWCols), kId1 = idesc_bf16(kCacheTile, kWBlock);
            const uint32_t q_atom = q_blocks * kWBlock * 128;
            uint32_t e = 0, loads = 0, steps[2] = {0, 0};
            bool ok = true, issued = false;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = ok && wait_bar(bar, parity, abort_flag, a.status, a.wait_cycles);
                return ok;
            };
            while (ok && w.next(a)) {
                const int R = w.s.n * a.rep;
                for (int r0 = 0; ok && r0 < R; r0 += kWRows) {
                    if (!wait(q_full, loads++ & 1)) break;
                    const int blocks = (min(kWRows, R - r0) + kWBlock - 1) / kWBlock;
                    for (int tile = w.tile0; ok && tile < w.tile1; ++tile, ++e) {
                        const int slot = (int)(e % n_stages);
                        if (!wait(&full[slot], (e / n_stages) & 1)) break;
                        const uint32_t ka = smem_u32(ring + slot * S::kTileBytes);
                        const int gr = (tile - w.tile0) & 1;
                        for (int k = 0; k < blocks; k += 2) {
                            const uint32_t n = steps[gr]++, buf = n % kWBufs, use = n / kWBufs;
                            if (use >= 1 && !wait(&s_empty[gr * kWBufs + buf], (use - 1) & 1)) break;
                            tc_fence_after();
                            issued = true;
                            const uint32_t to = tmem + (gr * kWBufs + buf) * kWCols, qa = smem_u32(sm + S::kQOff) + k * kWBlock * 128;
                            if (k + 1 < blocks)
                                product_k_major<kId2, D>(to, ka, kAtom, qa, q_atom);
                            else
                                product_k_major<kId1, D>(to, ka, kAtom, qa, q_atom);
                            mma_commit(&s_full[gr * kWBufs + buf]);
                        }
                        if (ok) mma_commit(&empty[slot]);
                    }
                }
            }
            if (issued) {
                mma_commit(drain);
                drain_wait(drain, 0, a.status);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------- epilogue
        const int gr = (warp - 2) >> 2, q = warp & 3, j = q * 32 + lane, tid = threadIdx.x - 64;
        float* fs = reinterpret_cast<float*>(sm + S::kFOff);
        uint32_t* nz = reinterpret_cast<uint32_t*>(sm + S::kNzOff);
        const uint32_t q_atom = q_blocks * kWBlock * 128;  // Q: [D / 64][rows] of 128 bytes
        uint32_t step = 0;
        bool alive = true;
        const bool lost = *a.timed_out != 0;  // the factors are not all there: no weight is written
        while (alive && w.next(a)) {
            const int R = w.s.n * a.rep;
            const int64_t row0 = a.cu[w.b];
            for (int r0 = 0; alive && r0 < R; r0 += kWRows) {
                const int nr = min(kWRows, R - r0), blocks = (nr + kWBlock - 1) / kWBlock;
                // Q and factors of this pass's rows; every S of the pass before is done with them
#pragma unroll 4
                for (int x = tid; x < blocks * kWBlock * (D / 8); x += 256) {
                    const int r = x / (D / 8), ch = x % (D / 8);
                    const int rr = r < nr ? r0 + r : r0, i = rr / a.rep, h = w.g * a.rep + rr % a.rep;
                    const char* from = a.Q + (row0 + i) * a.ldq + (int64_t)h * (D * 2) + ch * 16;
                    const uint32_t at = smem_u32(sm + S::kQOff) + (ch >> 3) * q_atom + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(r < nr ? 16 : 0)
                                 : "memory");
                }
                for (int r = tid; r < blocks * kWBlock; r += 256) {  // whole warps
                    float2 f = make_float2(0.f, 0.f);
                    if (r < nr && a.row_inside(row0 + (r0 + r) / a.rep)) f = a.factor[(row0 + (r0 + r) / a.rep) * a.Hq + w.g * a.rep + (r0 + r) % a.rep];
                    fs[(r >> 1) * 4 + (r & 1)] = f.x;
                    fs[(r >> 1) * 4 + 2 + (r & 1)] = f.y;
                    const uint32_t bits = __ballot_sync(0xffffffffu, f.y != 0.f);
                    if (lane == 0) nz[r >> 5] = bits;
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                both_groups_or(false);  // the factors are everyone's
                if (lane == 0) mbar_arrive(q_full);
                for (int tile = w.tile0 + gr; tile < w.tile1; tile += 2) {
                    const bool drafts = tile == w.s.nt - 1;
                    const int keys = tile_keys(a, w.s, tile);
                    float* to = nullptr;
                    float had = 0.f;
                    if (j < keys) {  // early: its latency passes under the sums
                        if (drafts) {
                            if (a.row_inside(row0 + j)) {
                                to = a.w_new + (row0 + j) * a.c.Hkv + w.g;
                                if (r0 > 0) had = *to;
                            }
                        } else {
                            const int slot = tile * kCacheTile + j;
                            const int64_t page = a.c.page_of(w.b, slot, a.status);
                            if (page >= 0 && a.c.inside(page, slot, w.g, a.status)) {
                                to = a.c.weight + a.c.meta(page, slot, w.g);
                                had = *to;
                            }
                        }
                    }
                    float2 sum[2] = {};
                    for (int k = 0; k < blocks; ++k) {
                        const uint32_t buf = step % kWBufs;
                        if (!(k & 1)) {
                            if (alive)
                                alive = warp_wait(&s_full[gr * kWBufs + buf], (step / kWBufs) & 1, abort_flag, a.status, a.wait_cycles);
                            tc_fence_after();
                        }
                        const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16) + (gr * kWBufs + buf) * kWCols + (k & 1) * kWBlock;
                        const int cols = min(kWBlock, nr - k * kWBlock);
                        uint64_t seen = (uint64_t)nz[2 * k + 1] << 32 | nz[2 * k];  // none past the rows
                        if (drafts) seen &= rows_that_see(a, row0, keys, j, r0 + k * kWBlock, cols);
                        float z[kWBlock];
                        tmem_ld32(ta, z);
                        tmem_ld32(ta + 32, z + 32);
                        tmem_wait_ld();
                        tie<kWBlock>(z);
                        if ((k & 1) || k + 1 == blocks) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&s_empty[gr * kWBufs + buf]);
                            ++step;
                        }
                        const float4* f4 = reinterpret_cast<const float4*>(fs + k * kWBlock * 2);
                        const float2 c2 = make_float2(a.scale_log2, a.scale_log2);
                        if (__all_sync(0xffffffffu, seen == ~0ull)) {
#pragma unroll
                            for (int i = 0; i < kWBlock; i += 2) {
                                const float4 f = f4[i / 2];
                                const float2 y = __ffma2_rn(make_float2(z[i], z[i + 1]), c2, make_float2(f.x, f.y));
                                sum[i / 2 & 1] = __ffma2_rn(make_float2(ex2(y.x), ex2(y.y)), make_float2(f.z, f.w), sum[i / 2 & 1]);
                            }
                        } else {
#pragma unroll
                            for (int c = 0; c < kWBlock; c += 16) {
                                if (c >= cols) break;
#pragma unroll
                                for (int i = c; i < c + 16; i += 2) {
                                    const float4 f = f4[i / 2];
                                    const float2 y = __ffma2_rn(make_float2(z[i], z[i + 1]), c2, make_float2(f.x, f.y));
                                    float2& s2 = sum[i / 2 & 1];
                                    if (seen >> i & 1) s2.x = fmaf(ex2(y.x), f.z, s2.x);
                                    if (seen >> i & 2) s2.y = fmaf(ex2(y.y), f.w, s2.y);
                                }
                            }
                        }
                    }
                    if (to != nullptr && alive && !lost) *to = had + ((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
                }
                if (both_groups_or(!alive)) alive = false;  // Q and the factors are free
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && *abort_flag) *a.timed_out = 1;
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kWBufs * kWCols));
    }
}

}  // namespace

estp_status launch_cache_weight_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st) {
    TcMaps tm;
    int box_rows, new_rows;
    const estp_status s = make_maps(a, &tm, &box_rows, &new_rows);
    if (s != ESTP_OK) return s;
    auto kernel = a.c.d == 128 ? cache_weight_tc_kernel<128> : cache_weight_tc_kernel<64>;
    const int rows = a.max_rows * a.rep < kWRows ? a.max_rows * a.rep : kWRows, blocks = (rows + kWBlock - 1) / kWBlock;
    const int smem = a.c.d == 128 ? WShape<128>::smem(blocks) : WShape<64>::smem(blocks);
    const int stages = a.c.d == 128 ? WShape<128>::stages(blocks) : WShape<64>::stages(blocks);
    cudaError_t e = set_smem(ctx, a.c.d == 128 ? 31 : 30, kernel, 227 * 1024);
    if (e != cudaSuccess) return cuda_fail(e, "cache weight smem attribute");
    e = launch_dependent(kernel, ctx->num_sms, WShape<128>::kThreads, (size_t)smem, st, tm, a, box_rows, new_rows, blocks, stages);
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache weight launch");
}

}  // namespace estp
