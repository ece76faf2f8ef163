// The forward half of the cache attention (see cache_attn.cu) for bf16 caches and more than 32 rows a
// (sequence, KV head), as wide draft trees give: the rows take the 128 lanes of an MMA.
//   S = Q K^T          M = 128 rows, N = 128 keys, K = D, into TMEM
//   P = 2^(S c - m)    a thread a row: the running maximum and sum need no exchange between lanes.
//                      Each P is two bf16 terms, hi + lo (16 bits of it enter the second product), written
//                      over the S that they come from: of every 32 columns, 16 of hi and 16 of lo
//   O += hi V + lo V   A = P from TMEM, B = the V tile as it is stored (MN-major), into TMEM
// (With the keys on the lanes, as cache_attn_tc.cu has them, 64 rows are 64 columns a thread: their
// maxima over the lanes, l and P in registers cost 2.4 us a tile where the copies need 1.45.)
//
// A row's m only moves when a tile exceeds it by 2^8; the warps whose rows do then rescale O and l.
//
// One persistent CTA per SM over the units of cache.cuh, two epilogue groups of 128 threads, each with
// an S/P buffer and an O of 128 columns (all 512).  A block of up to 128 rows is split by tiles: the groups
// take them in turn, each with a softmax of its own, and are joined at a segment's end.  A block of up
// to 256 rows is split by rows, 128 a group, and every tile goes to both.  Either way one group's
// softmax runs under the other's products.
//   warps 0, 2 TMA producers of the K and of the V tiles, a ring each
//   warps 1, 3 issue the products of a group each; the pipe runs a warp's in the order of issue, so the
//              S that overwrites a P comes after the product that reads it.  A tile's slot is free when
//              both have let go of it.  (One warp for both groups held each back for the other: 178 us
//              against 152 for 8 sequences of 8k with 9 to 17 drafts, 8 query heads a KV head.)
//   warps 4-11 the epilogue groups, which also load their rows' Q.  The second half of the keys is
//              handed on first, so that its product runs under the first half's exponentials (152 to
//              148 us).  Two warps to a group's 32 rows have 96 registers a thread: 198 us.
// Bound by the turn of a group: 1.5 us of softmax and 1.6 of products (24 of 64 clocks, the other
// group's between them) for every tile, 1.55 us a tile with two groups, where the tensor pipe needs 0.85
// and the copies 1.45.  Another S buffer would part them.  At head size 128 the columns are spent; at 64 an
// O takes half of the columns kept for it, and a third S buffer would fit: it is not built.
// Keys past a sequence's slots, drafts that are not finite and waits are treated as in
// cache_attn_tc.cu.
#include "cache_tc.cuh"

namespace estp {
namespace {

template <int D>
struct RowShape {
    static constexpr int kAtoms = D / 64;
    static constexpr int kTileBytes = kAtoms * kAtom;  // 128 keys, or 128 rows of Q
    static constexpr int kMaxStages = 12;
    static constexpr int kThreads = 384;
    // from a 1024-aligned base: barriers and flags, Q (one tile of rows or two), the ring
    static constexpr int kBars = 2 * kMaxStages + 12;
    static constexpr int kMiscOff = (kBars * 8 + 15) / 16 * 16;  // tmem address, abort flag, tiles issued, odd drafts
    static constexpr int kQOff = 1024;
    static_assert(kMiscOff + 48 <= kQOff, "barriers");
    static int stages(int q_tiles) {
        const int n = (227 * 1024 - 1024 - kQOff) / kTileBytes - q_tiles;
        return n < kMaxStages ? n : kMaxStages;
    }
    static int smem(int q_tiles) { return 1024 + kQOff + (q_tiles + stages(q_tiles)) * kTileBytes; }
};

// D (TMEM) += A (TMEM) B, B an MN-major shared memory tile
template <uint32_t kIdesc>
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b), "r"(kIdesc), "r"(acc));
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

template <int D>
__global__ void __launch_bounds__(RowShape<D>::kThreads, 1)
    cache_rows_tc_kernel(const __grid_constant__ TcMaps tm, const CacheAttnArgs a, const int box_rows, const int new_rows,
                         const int n_stages) {
    using S = RowShape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
    uint8_t* ring = sm + S::kQOff + (a.RB / 128) * S::kTileBytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm);  // [kMaxStages], K then V
    uint64_t* empty = full + S::kMaxStages;            // [kMaxStages]
    const int k_stages = n_stages / 2;                 // V tiles wait longer in their slots
    const Ring ring_k{full, empty, ring, k_stages, S::kTileBytes};
    const Ring ring_v{full + k_stages, empty + k_stages, ring + k_stages * S::kTileBytes, n_stages - k_stages, S::kTileBytes};
    uint64_t* q_full = empty + S::kMaxStages;          // [2] a group's rows, a phase a segment that has a tile for it
    uint64_t* s_full = q_full + 2;                     // [2]
    uint64_t* p_full = s_full + 2;                     // [2][2] halves of the keys
    uint64_t* o_full = p_full + 4;                     // [2]
    uint64_t* drain = o_full + 2;                      // [2]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + S::kMiscOff);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::kMiscOff + 4);
    volatile int* issued_tiles = reinterpret_cast<volatile int*>(sm + S::kMiscOff + 8);  // [2] K, V
    volatile uint32_t* odd = reinterpret_cast<volatile uint32_t*>(sm + S::kMiscOff + 16);  // [2][4] drafts with V not finite

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < n_stages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 2);  // both issuers
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 8);  // the epilogue warps
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[2 * i], 4);
            mbar_init(&p_full[2 * i + 1], 4);
            mbar_init(&o_full[i], 1);
        }
        mbar_init(&drain[0], 1);
        mbar_init(&drain[1], 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    await_stream();
    const uint32_t tmem = *tmem_slot;
    const int cta = blockIdx.x;
    Walk walk{Place{0, 0, 0, 0}, 0, 0};
    Place place;
    const PlanTotals tot = plan(a, reinterpret_cast<PlanScratch*>(ring), &place, [&](const Place& x, const SeqShape& s, const PlanTotals& all) {
        const int u = share_begin(cta, all.units, ctas_of(a, all.units));
        return u >= x.unit0 && u < x.unit0 + s.units(a.c.Hkv);
    });
    const int G = ctas_of(a, tot.units);
    if (tot.ok && cta < G) walk = Walk{place, share_begin(cta, tot.units, G), share_begin(cta + 1, tot.units, G)};
    if (a.B > 32) {  // the plan used its scratch, in the ring
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    Segment sg;

    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------ producers
        const int kv = warp == 2;
        const Ring mine = kv ? ring_v : ring_k;
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(
                          kv ? (lane ? &tm.vn : &tm.v) : (lane ? &tm.kn : &tm.k))) : "memory");
        uint32_t t = 0;
        bool ok = true;
        PageWindow win;
        while (ok && walk.next(a, sg)) {
            win.open(a, sg.s, sg.b, sg.tile0, lane);
            for (int tile = sg.tile0; tile < sg.tile1; ++tile, ++t) {
                if (t >= (uint32_t)mine.n && !warp_wait(mine.freed(t), mine.parity(t - mine.n), abort_flag, a.status, a.wait_cycles)) {
                    ok = false;
                    break;
                }
                load_tile<D>(a, kv ? &tm.v : &tm.k, kv ? &tm.vn : &tm.kn, win, sg.s, sg.b, sg.g, tile, box_rows, new_rows,
                             mine.tile(t), mine.filled(t), lane);
            }
        }
        if (lane == 0) issued_tiles[kv] = (int)t;
        __syncwarp();
    } else if (warp < 4) {
        // --------------------------------------------------------- MMA issuers
        if (lane == 0) {
            constexpr uint32_t kIdS = idesc_bf16(128, 128);
            constexpr uint32_t kIdO = idesc_bf16(128, D) | (1u << 16);  // B MN-major
            const int w = warp >> 1;  // the group
            const uint32_t sp = tmem + w * 128, o = tmem + 256 + w * 128;
            uint32_t t = 0, q_seen = 0, p_seen = 0;
            bool ok = true, issued = false;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = ok && wait_bar(bar, parity, abort_flag, a.status, a.wait_cycles);
                return ok;
            };
            while (ok && walk.next(a, sg)) {
                const int tiles = sg.tile1 - sg.tile0;
                const bool split = sg.nr <= 128;  // by tiles; else by rows
                const int first = split ? w : 0, step = split ? 2 : 1;
                int k_at = 0, v_at = 0;  // tiles that this issuer is done with
                bool live = false;
                // Q is awaited where the group has a tile, and only there is its barrier arrived at: a phase that this
                // warp let pass would leave it a parity behind, on which the next wait is over before Q is there
                if (first < tiles && !wait(&q_full[w], q_seen++ & 1)) break;
                auto pass = [&](const Ring& r, int& at, int to) {  // the other group's tiles
                    for (; ok && at < to; ++at)
                        if (wait(r.filled(t + at), r.parity(t + at))) mbar_arrive(r.freed(t + at));
                };
                auto product_s = [&](int i) {  // S of the segment's tile i
                    pass(ring_k, k_at, i);
                    if (!wait(ring_k.filled(t + i), ring_k.parity(t + i))) return;
                    tc_fence_after();
                    issued = true;
                    product_k_major<kIdS, D>(sp, smem_u32(sm + S::kQOff) + (split ? 0 : w * S::kTileBytes), kAtom,
                                             smem_u32(ring_k.tile(t + i)), kAtom);
                    mma_commit(&s_full[w]);
                    mma_commit(ring_k.freed(t + i));
                    k_at = i + 1;
                };
                auto product_o = [&](int i) {
                    pass(ring_v, v_at, i);
                    if (!wait(ring_v.filled(t + i), ring_v.parity(t + i)) || !wait(&p_full[2 * w + 1], p_seen & 1)) return;
                    tc_fence_after();
                    issued = true;
                    const int ksteps = (tile_keys(a, sg.s, sg.tile0 + i) + 15) / 16;
                    const uint64_t vd = mn_desc(smem_u32(ring_v.tile(t + i)), kAtom);
                    auto keys16 = [&](int kk, uint32_t acc) {  // 16 keys, 2 KB of V: hi and lo
                        const uint32_t at = sp + (kk >> 1) * 32 + (kk & 1) * 8;
                        mma_ts<kIdO>(o, at, vd + kk * 128, acc);
                        mma_ts<kIdO>(o, at + 16, vd + kk * 128, 1u);
                    };
                    if (ksteps == 8) {
#pragma unroll
                        for (int kk = 4; kk < 8; ++kk) keys16(kk, kk > 4 ? 1u : live ? 1u : 0u);
                        if (!wait(&p_full[2 * w], p_seen++ & 1)) return;
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) keys16(kk, 1u);
                    } else {
                        if (!wait(&p_full[2 * w], p_seen++ & 1)) return;
                        tc_fence_after();
                        for (int kk = 0; kk < ksteps; ++kk) keys16(kk, live || kk > 0 ? 1u : 0u);
                    }
                    live = live || ksteps > 0;
                    if (i + step >= tiles) mma_commit(&o_full[w]);
                    mma_commit(ring_v.freed(t + i));
                    v_at = i + 1;
                };
                if (first < tiles) product_s(first);
                for (int i = first; ok && i < tiles; i += step) {
                    product_o(i);
                    if (ok && i + step < tiles) product_s(i + step);
                }
                pass(ring_k, k_at, tiles);
                pass(ring_v, v_at, tiles);
                t += tiles;
            }
            if (issued) {
                mma_commit(&drain[w]);
                drain_wait(&drain[w], 0, a.status);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------- epilogue
        const int w = (warp - 4) >> 2, q = warp & 3;
        const int j = q * 32 + lane;  // lane of TMEM: row of the group; and V row that it may clear
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t t_s = tmem + lane_off + w * 128, t_o = tmem + lane_off + 256 + w * 128;
        uint32_t t = 0, steps = 0, ends = 0;
        bool alive = true;
        auto wait = [&](uint64_t* b, uint32_t parity) {
            if (alive) alive = warp_wait(b, parity, abort_flag, a.status, a.wait_cycles);
        };
        while (walk.next(a, sg)) {
            const int tiles = sg.tile1 - sg.tile0;
            const bool split = sg.nr <= 128;
            const int base = split ? 0 : w * 128;
            volatile uint32_t* odd_drafts = odd + (split ? w : 0) * 4;
            const int64_t row0 = a.cu[sg.b];
            {  // Q (zeros past the rows), K-major with the 128-byte swizzle
                const uint32_t to = smem_u32(sm + S::kQOff);
                constexpr int kTogether = 256 / (D / 8);  // rows at a time
                const int x = w * 128 + j, ch = x % (D / 8);
                int i = (sg.r0 + x / (D / 8)) / a.rep, h = (sg.r0 + x / (D / 8)) % a.rep;
#pragma unroll 2
                for (int r = x / (D / 8); r < (split ? 128 : 256); r += kTogether) {
                    const bool there = r < sg.nr;
                    const char* from = a.Q + ch * 16;
                    if (there) from += (row0 + i) * a.ldq + (int64_t)(sg.g * a.rep + h) * (D * 2);
                    for (h += kTogether; h >= a.rep; h -= a.rep) ++i;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                     to + (r >> 7) * S::kTileBytes + (ch >> 3) * kAtom + (r & 127) * 128 + (((ch & 7) ^ (r & 7)) << 4)),
                                 "l"(from), "r"(there ? 16 : 0)
                                 : "memory");
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&q_full[0]);
                    if (!split || tiles > 1) mbar_arrive(&q_full[1]);
                }
            }
            const int rr = sg.r0 + base + j;  // this thread's row of the (b, KV head)
            const bool mine = base + j < sg.nr;
            const int draft = mine ? rr / a.rep : 0;
            float m = -INFINITY, l = 0.f;
            bool live = false;
            const float c = a.scale_log2;
            const int first = sg.tile0 + (split ? w : 0);
            for (int tile = first; tile < sg.tile1; tile += split ? 2 : 1, ++steps) {
                const bool drafts = tile == sg.s.nt - 1;
                const int keys = tile_keys(a, sg.s, tile);
                uint64_t seen[2] = {~0ull, ~0ull};  // keys that this row sees
                if (drafts) {
                    if (a.tree != nullptr) {
                        const uint64_t* p = a.tree + (row0 + draft) * a.words;
                        seen[0] = p[0];
                        seen[1] = a.words > 1 ? p[1] : 0;
                    } else {
                        seen[0] = draft >= 63 ? ~0ull : (1ull << (draft + 1)) - 1;
                        seen[1] = draft >= 127 ? ~0ull : draft < 64 ? 0 : (1ull << (draft - 63)) - 1;
                    }
                }
                if (keys < kCacheTile) {
                    seen[0] &= keys >= 64 ? ~0ull : (1ull << keys) - 1;
                    seen[1] &= keys <= 64 ? 0 : (1ull << (keys - 64)) - 1;
                }
                const bool masked = drafts || keys < kCacheTile;
                wait(&s_full[w], steps & 1);
                tc_fence_after();
                float z[64];
                auto load = [&](int half) {  // 64 keys of S, hidden ones at -inf
                    tmem_ld32(t_s + half * 64, z);
                    tmem_ld32(t_s + half * 64 + 32, z + 32);
                    tmem_wait_ld();
                    tie<64>(z);
                    if (masked) {
                        const uint64_t bits = seen[half];
#pragma unroll
                        for (int k = 0; k < 64; ++k)
                            if (!(bits >> k & 1)) z[k] = -INFINITY;
                    }
                };
                float top = -INFINITY;
                auto highest = [&]() {
                    float t4[4] = {top, z[0], z[1], z[2]};
#pragma unroll
                    for (int k = 3; k < 63; k += 8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (k + 2 * i + 1 < 64) t4[i] = fmax3(t4[i], z[k + 2 * i], z[k + 2 * i + 1]);
                    }
                    top = fmaxf(fmax3(t4[0], t4[1], z[63]), fmaxf(t4[2], t4[3]));
                };
                load(0);
                highest();
                load(1);
                highest();
                // m moves when the tile exceeds it by 2^8 (always where there is none)
                const float high = top * c;
                float f = 1.f;
                if (high > m + 8.f) {
                    f = ex2(m - high);
                    m = high;
                }
                l *= f;
                if (__any_sync(0xffffffffu, f != 1.f) && live) {
#pragma unroll 1
                    for (int x = 0; x < D; x += 32) {
                        float o[32];
                        tmem_ld32(t_o + x, o);
                        tmem_wait_ld();
                        tie<32>(o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] *= f;
                        tmem_st32(t_o + x, reinterpret_cast<const uint32_t*>(o));
                    }
                }
                const float nm = m == -INFINITY ? 0.f : -m;
                float2 sum = make_float2(0.f, 0.f);
                auto exponentials = [&](int half) {
                    const float2 c2 = make_float2(c, c), n2 = make_float2(nm, nm);
#pragma unroll
                    for (int x = 0; x < 64; x += 32) {
                        uint32_t p[32];
#pragma unroll
                        for (int k = 0; k < 32; k += 2) {
                            const float2 y = __ffma2_rn(make_float2(z[x + k], z[x + k + 1]), c2, n2);
                            const float2 e = make_float2(ex2(y.x), ex2(y.y));
                            sum = __fadd2_rn(sum, e);
                            p[k / 2] = pack_hi_lo(e.x, e.y, p[16 + k / 2]);
                        }
                        tmem_st32(t_s + half * 64 + x, p);
                    }
                };
                const bool unsound = drafts || (keys & 15);
                if (unsound && (split || w == 0)) {
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
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (unsound && !split) both_groups_or(false);  // both groups' products read the cleared rows
                auto half_done = [&](int half) {
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[2 * w + half]);
                };
                exponentials(1);  // still in registers
                half_done(1);
                load(0);
                exponentials(0);
                l += sum.x + sum.y;
                half_done(0);
                live = live || keys > 0;
            }
            t += tiles;
            if (first < sg.tile1) wait(&o_full[w], ends++ & 1);  // the last product of the segment
            const bool whole = sg.tile0 == 0 && sg.tile1 == sg.s.nt;
            if (both_groups_or(!alive)) break;  // the groups leave together
            tc_fence_after();
            // drafts whose V is not finite were left out of O; their P is still in its place
            if (sg.tile1 == sg.s.nt && (!split || ((tiles - 1) & 1) == w) &&
                (odd_drafts[0] | odd_drafts[1] | odd_drafts[2] | odd_drafts[3])) {
#pragma unroll 1
                for (int x = 0; x < sg.s.n; ++x) {
                    if (!(odd_drafts[x >> 5] >> (x & 31) & 1)) continue;
                    const bool sees = mine && (a.tree != nullptr ? a.tree[(row0 + draft) * a.words + (x >> 6)] >> (x & 63) & 1 : x <= draft);
                    uint32_t hi, lo;
                    const uint32_t at = t_s + (x >> 5) * 32 + ((x & 31) >> 1);
                    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(hi) : "r"(at));
                    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(lo) : "r"(at + 16));
                    tmem_wait_ld();
                    asm volatile("" : "+r"(hi), "+r"(lo));
                    const float p = x & 1 ? bf16hi(hi) + bf16hi(lo) : bf16lo(hi) + bf16lo(lo);
                    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(a.vn + (row0 + x) * a.ldn + (int64_t)sg.g * (D * 2));
#pragma unroll 1
                    for (int y = 0; y < D; y += 16) {
                        float o[16];
                        tmem_ld16(t_o + y, o);
                        tmem_wait_ld();
                        tie<16>(o);
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (sees) o[k] = fmaf(p, __bfloat162float(v[y + k]), o[k]);
                        tmem_st16(t_o + y, o);
                    }
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                }
            }
            const int h = sg.g * a.rep + rr % a.rep;
            const int64_t row = row0 + draft;
            // split by tiles: joined with the other group's half, which lies on the same lanes
            float M = m, L = l, fa = live ? 1.f : 0.f, fb = 0.f;
            if (split) {
                float2* ml = reinterpret_cast<float2*>(sm + S::kQOff);  // [2][128]: every S is done with Q
                ml[w * 128 + j] = make_float2(m, l);
                tc_fence_before();
                both_groups_or(false);
                tc_fence_after();
                const float2 o = ml[(1 - w) * 128 + j];
                M = fmaxf(m, o.x);
                fa = m == -INFINITY ? 0.f : ex2(m - M);
                fb = o.x == -INFINITY ? 0.f : ex2(o.x - M);
                const float la = fa != 0.f ? fa * l : M == -INFINITY ? l : 0.f, lb = fb != 0.f ? fb * o.y : M == -INFINITY ? o.y : 0.f;
                L = w == 0 ? la + lb : lb + la;
                if (L != L) fa = fb = 1.f;  // NaN stays
            }
            const float scale = !whole ? 1.f : M == -INFINITY && L == 0.f ? 0.f : 1.f / L;
            fa *= scale;
            fb *= scale;
            const int64_t part = (int64_t)(cta + sg.group) * a.RB + base + j;
            const bool inside = !mine || (whole ? a.row_inside(row) : a.part_inside(cta + sg.group));
            if (mine && inside && (!split || w == 0)) {
                if (!whole) a.part_ml[part] = make_float2(M, L);
                if (whole && a.lse != nullptr) a.lse[(int64_t)h * a.n_rows + row] = L == 0.f ? -INFINITY : fmaf(M, kLn2, logf(L));
                if (whole && a.factor != nullptr) a.factor[row * a.Hq + h] = weight_factor(a, make_float2(M, L), row);
            }
            // split by tiles: each group writes half of the columns
            const uint32_t t_b = tmem + lane_off + 256 + (1 - w) * 128;
            const int cols = split ? D / 2 : D, x0 = split ? w * cols : 0;
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.out) + (row * a.Hq + h) * D;
#pragma unroll 1
            for (int x = x0; x < x0 + cols; x += 16) {
                float o[16], b[16];
                tmem_ld16(t_o + x, o);
                tmem_ld16(t_b + x, b);
                tmem_wait_ld();
                tie<16>(o);
                tie<16>(b);
                if (!mine || !inside) continue;
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    o[k] = fa != 0.f ? o[k] * fa : 0.f;
                    if (fb != 0.f) o[k] = fmaf(b[k], fb, o[k]);
                }
                if (whole) {
                    uint32_t v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const __nv_bfloat162 t2 = __floats2bfloat162_rn(o[2 * k], o[2 * k + 1]);
                        v[k] = *reinterpret_cast<const uint32_t*>(&t2);
                    }
                    *reinterpret_cast<uint4*>(out + x) = make_uint4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<uint4*>(out + x + 8) = make_uint4(v[4], v[5], v[6], v[7]);
                } else {
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        *reinterpret_cast<float4*>(a.part_o + part * D + x + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                }
            }
            tc_fence_before();
            both_groups_or(false);  // Q and O are free for the next segment
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    admit_next();
    if (threadIdx.x == 0 && *abort_flag) {
        *a.timed_out = 1;  // the partials and scores are not all there
        ring_k.drain(issued_tiles[0], a.status);
        ring_v.drain(issued_tiles[1], a.status);
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

template <int D>
estp_status launch(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st) {
    using S = RowShape<D>;
    TcMaps tm;
    int box_rows, new_rows;
    const estp_status s = make_maps(a, &tm, &box_rows, &new_rows);
    if (s != ESTP_OK) return s;
    cudaError_t e = set_smem(ctx, D == 128 ? 21 : 20, cache_rows_tc_kernel<D>, 227 * 1024);
    if (e != cudaSuccess) return cuda_fail(e, "cache attention smem attribute");
    const int q_tiles = a.RB / 128;
    e = launch_dependent(cache_rows_tc_kernel<D>, a.G, S::kThreads, (size_t)S::smem(q_tiles), st, tm, a, box_rows, new_rows, S::stages(q_tiles));
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache attention launch");
}

}  // namespace

estp_status launch_cache_rows_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st) {
    return a.c.d == 128 ? launch<128>(ctx, a, st) : launch<64>(ctx, a, st);
}

}  // namespace estp
