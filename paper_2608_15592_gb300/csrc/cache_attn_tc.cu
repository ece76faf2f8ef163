// The forward half of the cache attention (see cache_attn.cu) for bf16 caches, on the tensor cores.
//
// Decoding has few rows and many keys, so the keys take the 128 lanes of an MMA and the rows its
// columns: per tile of 128 keys and block of RB rows
//   S^T = K Q^T          M = 128 keys, N = RB, K = D
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
//   warps 0, 3 TMA producers of the K and of the V tiles, which take turns in one ring, a box a page
//              (a lane each); warp 3 also loads the rows' Q, up to 64 rows a segment ahead
//   warp 1     issues S, as far ahead as K tiles and S buffers allow
//   warp 2     issues O, as soon as a P is written
//   warps 4-11 two epilogue groups of 4 warps, each with its S (double-buffered) and O in tensor
//              memory and its P buffer; up to 64 rows they take the tiles in turn, more rows are
//              shared out between them
// Keys past a sequence's slots hold anything: S^T has them replaced, their P is 0 and their V rows
// (up to the MMA's 16-key step) are zeroed in shared memory before the product, as 0 x NaN is not 0.
// A draft whose V is not finite is zeroed there too and added by itself to the rows that see it.
//
// Bound by the K and V bytes while the rows cost less than the 64 KB of a tile take to arrive
// (1.45 us an SM at the copy rate).  Every wait is bounded; on expiry the CTA records
// ESTP_ERR_TIMEOUT, the group votes to leave, and copies and MMAs are drained before TMEM is freed.
#include "cache.cuh"
#include "tcgen05.cuh"

namespace estp {
namespace {

constexpr int kAtom = kCacheTile * 128;  // 128 keys x 64 bf16

// Two epilogue groups.  KS = 2: they take the tiles of a segment in turn, each with a softmax of its
// own over the block's RB rows (a group leaves a partial of its own).  KS = 1: every tile goes to
// both, group g owning rows g RB .. of a block of 2 RB.
constexpr int kGroups = 2;

template <int D, int RB, int KS>
struct Shape {
    static constexpr int kN = RB < 16 ? 16 : RB;  // S columns: an MMA of M = 128 has N >= 16
    static constexpr int kAtoms = D / 64;
    static constexpr int kTileBytes = kAtoms * kAtom;
    static constexpr int kQRows = KS == 2 ? kN : 2 * RB;          // rows of a block
    static constexpr int kQBufs = RB == 64 ? 1 : 2;               // two: the next segment's Q loads ahead
    static constexpr int kRowArrays = KS == 2 ? 5 : 3;            // [RB] floats a group keeps
    static constexpr int kQBytes = kAtoms * kQRows * 128;
    // P: [128 keys] rows of 128 bytes, hi then lo; 64 rows take two, up to 16 share one between the groups
    static constexpr int kPStep = RB == 64 ? 2 * kAtom : RB == 32 ? kAtom : 64;  // from a group's P to the other's
    static constexpr int kPBytes = RB == 64 ? 4 * kAtom : RB == 32 ? 2 * kAtom : kAtom;
    static constexpr int kFixed = kQBufs * kQBytes + kPBytes;
    static constexpr int kRoom = 227 * 1024 - 1024 - kFixed - 400 - kGroups * (kRowArrays + (RB == 64 ? 0 : 4)) * RB * 4;
    static constexpr int kStages = kRoom / kTileBytes < 12 ? kRoom / kTileBytes : 12;
    static constexpr int kThreads = 128 + 128 * kGroups;
    static constexpr int kTmemUsed = kGroups * (2 * kN + 2 * RB);  // S twice, O hi and lo
    static constexpr int kTmem = kTmemUsed <= 128 ? 128 : kTmemUsed <= 256 ? 256 : 512;
    static constexpr int kOCol = kGroups * 2 * kN;
    // offsets from a 1024-aligned base
    static constexpr int kPOff = kStages * kTileBytes;
    static constexpr int kQOff = kPOff + kPBytes;
    static constexpr int kRedOff = kQOff + kQBufs * kQBytes;   // a group's [4][RB] per-warp values
    // (64 rows: in the P buffer, when it is free)
    static constexpr int kBarOff = kRedOff + (RB == 64 ? 0 : kGroups * 4 * RB * 4);
    static constexpr int kBars = 2 * kStages + 2 * kQBufs + 6 * kGroups + 2;
    static constexpr int kMiscOff = kBarOff + (kBars * 8 + 15) / 16 * 16;  // tmem address, abort flag, poison bits
    static constexpr int kRowOff = kMiscOff + 48;  // a group's row arrays
    static constexpr int kSmem = kRowOff + kGroups * kRowArrays * RB * 4 + 1024;
    static_assert(kStages >= 4 && kSmem <= 227 * 1024, "shared memory per CTA");
};

// tcgen05.ld / .st of 16 or 32 fp32 columns of this thread's lane
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
    uint32_t r[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) r[k] = __float_as_uint(v[k]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* v) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, float* v) {
    uint32_t r[4];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(taddr));
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(r[k]);
}
template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, float* v) {
    if (N == 4) tmem_ld4(taddr, v);
    else if (N == 8) tmem_ld8(taddr, v);
    else tmem_ld16(taddr, v);
}
// Orders every later use of v[0..N) after the wait for the load that fills them.
template <int N>
__device__ __forceinline__ void tie(float* v) {
#pragma unroll
    for (int k = 0; k < N; k += 4) asm volatile("" : "+f"(v[k]), "+f"(v[k + 1]), "+f"(v[k + 2]), "+f"(v[k + 3]));
}

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
        : "memory");
}

// MN-major tile, 128-byte swizzle: 64 values of a key a 128-byte row, 8-key groups 1 KB apart, the
// second 64 values `lead` bytes on.
__device__ __forceinline__ uint64_t mn_desc(uint32_t addr, uint32_t lead) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// Barrier of one epilogue group (128 threads) that ors a predicate.
__device__ __forceinline__ bool group_or(int id, bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.aligned.pred q, %2, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)x), "r"(id)
        : "memory");
    return r != 0;
}
// The same for both groups.
__device__ __forceinline__ bool both_groups_or(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.aligned.pred q, 3, 256, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)x)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ void group_sync(int id) { asm volatile("barrier.cta.sync.aligned %0, 128;" ::"r"(id) : "memory"); }

__device__ __forceinline__ uint32_t pack_hi_lo(float a, float b, uint32_t& lo) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    const __nv_bfloat162 l = __floats2bfloat162_rn(a - __low2float(h), b - __high2float(h));
    lo = *reinterpret_cast<const uint32_t*>(&l);
    return *reinterpret_cast<const uint32_t*>(&h);
}

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

// A segment: consecutive tiles [tile0, tile1) of one (b, g, row block).
struct Segment {
    SeqShape s;
    int b, g, r0, nr, tile0, tile1;
    int group;
};
// Walks the segments of units [u, u1); every role of the CTA walks them by itself.
struct Walk {
    Place at;
    int u, u1;
    __device__ __forceinline__ bool next(const CacheAttnArgs& a, Segment& o) {
        while (u < u1) {
            o.s = seq_shape(a, at.b);
            if (u >= at.unit0 + o.s.units(a.c.Hkv)) {
                at.pass(o.s, a.c.Hkv);
                continue;
            }
            const int loc = u - at.unit0, grp = loc / o.s.nt;
            o.tile0 = loc % o.s.nt;
            o.tile1 = min(o.s.nt, o.tile0 + (u1 - u));
            o.b = at.b;
            o.g = grp / o.s.nrb;
            o.r0 = grp % o.s.nrb * a.RB;
            o.nr = min(a.RB, o.s.n * a.rep - o.r0);
            o.group = at.group0 + grp;
            u += o.tile1 - o.tile0;
            return true;
        }
        return false;
    }
};
// Keys of a tile that exist.
__device__ __forceinline__ int tile_keys(const CacheAttnArgs& a, const SeqShape& s, int tile) {
    if (tile == s.nt - 1) return a.kn != nullptr ? s.n : 0;
    return min(kCacheTile, s.len - tile * kCacheTile);
}

struct TcMaps {
    CUtensorMap k, v, kn, vn;
};

// The page table of a sequence as a producer warp reads it: 32 entries at a time, a lane each, the
// next 32 already on their way (looked up tile by tile, the table's latency was two thirds of a
// tile's time).
struct PageWindow {
    const int32_t* row;
    int last, base, cur, nxt;  // last page in use; page index of lane 0; entries
    __device__ __forceinline__ int load(int i) const { return i <= last ? row[i] : 0; }
    __device__ __forceinline__ void open(const CacheAttnArgs& a, const SeqShape& s, int b, int tile, int lane) {
        row = a.c.table + (int64_t)b * a.c.ld_table;
        last = (s.len - 1) >> a.c.shift;  // -1 without slots
        base = (int)((int64_t)tile * kCacheTile >> a.c.shift);
        cur = load(base + lane);
        nxt = load(base + 32 + lane);
    }
    // entry of page index i; first is the smallest of the warp's
    __device__ __forceinline__ int get(int first, int i, int lane) {
        while (first >= base + 32) {
            base += 32;
            cur = nxt;
            nxt = load(base + 32 + lane);
        }
        const int x = __shfl_sync(0xffffffffu, cur, (i - base) & 31), y = __shfl_sync(0xffffffffu, nxt, (i - base) & 31);
        return i - base < 32 ? x : y;
    }
};

// A producer warp's copies of one tile: a lane a box of box_rows slots (or one of new_rows drafts).
template <int D>
__device__ __forceinline__ void load_tile(const CacheAttnArgs& a, const CUtensorMap* pages, const CUtensorMap* rows,
                                          PageWindow& win, const SeqShape& s, int b, int g, int tile, int box_rows,
                                          int new_rows, uint8_t* to, uint64_t* bar, int lane) {
    const int keys = tile_keys(a, s, tile);
    if (tile == s.nt - 1) {
        if (lane == 0) {
            mbar_expect_tx(bar, keys > 0 ? (uint32_t)(new_rows * 2 * D) : 0u);
            if (keys > 0)
#pragma unroll
                for (int x = 0; x < D / 64; ++x) tma_load_3d(to + x * kAtom, rows, x * 64, g, a.cu[b], bar);
        }
    } else {
        const int boxes = (keys + box_rows - 1) / box_rows, slot = tile * kCacheTile + lane * box_rows;
        int page = win.get(tile * kCacheTile >> a.c.shift, slot >> a.c.shift, lane);
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)(boxes * box_rows * 2 * D));
        __syncwarp();
        if (lane < boxes) {
            if (page < 0 || page >= a.c.n_pages) {
                report(a.status, ESTP_ERR_INVALID_ARG);
                page = a.c.n_pages > 0 ? (int)a.c.n_pages : 1;  // past the pool: reads as zero
            }
            to += lane * box_rows * 128;
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
                tma_load_4d(to + x * kAtom, pages, x * 64, slot & ((1 << a.c.shift) - 1), g, page, bar);
        }
    }
    __syncwarp();
}

template <int D, int RB, int KS>
__global__ void __launch_bounds__(Shape<D, RB, KS>::kThreads, 1)
    cache_fwd_tc_kernel(const __grid_constant__ TcMaps tm, const CacheAttnArgs a, const int box_rows, const int new_rows) {
    using S = Shape<D, RB, KS>;
    constexpr int NB = kGroups;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + S::kBarOff);  // [kStages]
    uint64_t* empty = full + S::kStages;                            // [kStages]
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
    volatile uint32_t* poison = reinterpret_cast<volatile uint32_t*>(sm + S::kMiscOff + 16);  // [2][4] drafts with V not finite

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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
        // warp 0 the K tiles (even ring entries), warp 3 the V tiles (odd ones) and the rows' Q
        const int kv = warp == 3;
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(
                          kv ? (lane ? &tm.vn : &tm.v) : (lane ? &tm.kn : &tm.k))) : "memory");
        uint32_t t = 0, q_seg = 0;  // tiles issued; segments whose Q is loaded
        bool ok = true;
        Walk q_walk = walk;
        Segment qs;
        // Q of the next segment (zeros past its rows), K-major with the 128-byte swizzle
        auto load_q = [&]() {
            if (!q_walk.next(a, qs)) return;
            const uint32_t qb = q_seg % S::kQBufs, use = q_seg / S::kQBufs;
            if (use >= 1 && !warp_wait(&q_empty[qb], (use - 1) & 1, abort_flag, a.status, a.wait_cycles)) {
                ok = false;
                return;
            }
            ++q_seg;
            const int64_t row0 = a.cu[qs.b];
            const uint32_t to = smem_u32(sm + S::kQOff + qb * S::kQBytes);
#pragma unroll 4
            for (int x = lane; x < S::kQRows * (D / 8); x += 32) {
                const int r = x / (D / 8), ch = x % (D / 8);
                const int rr = r < qs.nr ? qs.r0 + r : qs.r0, i = rr / a.rep, h = qs.g * a.rep + rr % a.rep;
                const char* from = a.Q + (row0 + i) * a.ldq + (int64_t)h * (D * 2) + ch * 16;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                 to + (ch >> 3) * S::kQRows * 128 + r * 128 + (((ch & 7) ^ (r & 7)) << 4)),
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
        while (ok && walk.next(a, sg)) {
            win.open(a, sg.s, sg.b, sg.tile0, lane);
            for (int tile = sg.tile0; tile < sg.tile1; ++tile, ++t) {
                const uint32_t e = 2 * t + kv, use = e / S::kStages;
                const int slot = (int)(e % S::kStages);
                if (use >= 1 && !warp_wait(&empty[slot], (use - 1) & 1, abort_flag, a.status, a.wait_cycles)) {
                    ok = false;
                    break;
                }
                load_tile<D>(a, kv ? &tm.v : &tm.k, kv ? &tm.vn : &tm.kn, win, sg.s, sg.b, sg.g, tile, box_rows, new_rows,
                             sm + slot * S::kTileBytes, &full[slot], lane);
                if (kv && S::kQBufs == 2 && tile == sg.tile0) load_q();  // a failure shows at the next wait
            }
            if (ok && kv && S::kQBufs == 1) load_q();
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
            while (ok && walk.next(a, sg)) {
                const int groups = (sg.nr + RB - 1) / RB, tiles = sg.tile1 - sg.tile0;
                const uint32_t qb = seg % S::kQBufs;
                if (!wait(&q_full[qb], (seg / S::kQBufs) & 1)) break;
                ++seg;
                for (int i = 0; ok && i < tiles; ++i, ++t) {
                    const uint32_t e = 2 * t;
                    const int slot = (int)(e % S::kStages);
                    if (!wait(&full[slot], (e / S::kStages) & 1)) break;
                    const uint32_t ka = smem_u32(sm + slot * S::kTileBytes);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        if (KS == 2 ? (i & 1) != nb : nb >= groups) continue;
                        const uint32_t n = steps[nb]++, buf = n & 1, use = n >> 1;
                        if (use >= 1 && !wait(&s_empty[2 * nb + buf], (use - 1) & 1)) break;
                        tc_fence_after();
                        issued = true;
                        const uint32_t qa = smem_u32(sm + S::kQOff + qb * S::kQBytes + (KS == 2 ? 0 : nb * RB * 128));
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk)
                            mma_bf16<kIdS>(tmem + (2 * nb + buf) * S::kN, sw128_desc(ka + (kk >> 2) * kAtom + (kk & 3) * 32),
                                           sw128_desc(qa + (kk >> 2) * S::kQRows * 128 + (kk & 3) * 32), kk > 0 ? 1u : 0u);
                        mma_commit(&s_full[2 * nb + buf]);
                    }
                    if (ok) mma_commit(&empty[slot]);
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
            while (ok && walk.next(a, sg)) {
                const int groups = (sg.nr + RB - 1) / RB, tiles = sg.tile1 - sg.tile0;
                bool live[NB] = {};  // a group's O holds a product of this segment
                for (int i = 0; ok && i < tiles; ++i, ++t) {
                    const uint32_t e = 2 * t + 1;
                    const int slot = (int)(e % S::kStages);
                    if (!wait(&full[slot], (e / S::kStages) & 1)) break;
                    const uint32_t va = smem_u32(sm + slot * S::kTileBytes);
                    const int ksteps = (tile_keys(a, sg.s, sg.tile0 + i) + 15) / 16;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        if (KS == 2 ? (i & 1) != nb : nb >= groups) continue;
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
                    if (ok) mma_commit(&empty[slot]);
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
        // [4][RB], used when the P buffer is free
        float* row_w = RB == 64 ? reinterpret_cast<float*>(pb + nb * S::kPStep)
                                : reinterpret_cast<float*>(sm + S::kRedOff) + nb * 4 * RB;
        // 16-byte chunk c of key k's P row of a group
        auto p_chunk = [&](int group, int k, int c) {
            if (RB == 64) return pb + group * S::kPStep + (c >> 3) * kAtom + k * 128 + (((c & 7) ^ (k & 7)) << 4);
            if (RB == 32) return pb + group * S::kPStep + k * 128 + ((c ^ (k & 7)) << 4);
            return pb + k * 128 + (((group * (S::kPStep / 16) + c) ^ (k & 7)) << 4);
        };
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t t_o = tmem + lane_off + (uint32_t)(S::kOCol + nb * 2 * RB);
        constexpr int kCols = RB < 16 ? 8 : 16;  // columns of a tensor memory load
        uint32_t step = 0, t = 0, seg = 0;
        bool alive = true;
        auto wait = [&](uint64_t* b, uint32_t parity) {
            if (alive) alive = warp_wait(b, parity, abort_flag, a.status, a.wait_cycles);
        };
        while (walk.next(a, sg)) {
            const int base = KS == 2 ? 0 : nb * RB, nr = min(RB, sg.nr - base);  // rows of this group
            // the drafts' poison bits: a group's own, or shared by both, of which group 0 may be a segment ahead
            volatile uint32_t* odd_drafts = poison + (KS == 2 ? nb : (int)(seg++ & 1)) * 4;
            if (nr <= 0) {                                // none: the other group works alone
                t += sg.tile1 - sg.tile0;
                continue;
            }
            const int64_t row0 = a.cu[sg.b];
            if (j < RB) row_m[j] = -INFINITY;
            float2 l[RB / 2];
#pragma unroll
            for (int r = 0; r < RB / 2; ++r) l[r] = make_float2(0.f, 0.f);
            bool live = false, lost = true;  // lost: a row has no m yet, every tile looks for one
            const int first = sg.tile0 + (KS == 2 ? nb : 0);
            const float2 c2 = make_float2(a.scale_log2, a.scale_log2);
            for (int tile = first; tile < sg.tile1; tile += KS, ++step) {
                const bool drafts = tile == sg.s.nt - 1;
                const int keys = tile_keys(a, sg.s, tile);
                const uint32_t buf = step & 1;
                uint64_t seen = ~0ull;  // rows that see this thread's key
                if (drafts) seen = rows_that_see(a, row0, keys, j, sg.r0 + base, nr);
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
                if (a.store && alive) {
                    float* to = a.score + ((int64_t)(walk.u - (sg.tile1 - tile)) * a.RB + base) * kCacheTile + j;
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
                    constexpr int kR = RB < 32 ? RB : 32;
                    const auto larger = [](float x, float y) { return fmaxf(x, y); };
#pragma unroll
                    for (int r = 0; r < RB; r += kR) {
                        const float x = reduce_scatter<kR>(z + r, lane, larger);
                        if (lane < kR) row_w[q * RB + r + lane] = x;
                    }
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
                if ((KS == 2 || nb == 0) && (drafts || (keys & 15))) {
                    // V rows that must not reach the product: past the keys, and drafts that are not finite
                    const uint32_t e = 2 * (t + (tile - sg.tile0)) + 1;
                    const int slot = (int)(e % S::kStages);
                    wait(&full[slot], (e / S::kStages) & 1);
                    uint8_t* vr = sm + slot * S::kTileBytes + j * 128;
                    bool clear = j >= keys && j < ((keys + 15) & ~15);
                    if (drafts && j < keys) {
                        bool odd = false;
#pragma unroll
                        for (int x = 0; x < S::kAtoms * 8; ++x) {
                            const uint4 v = *reinterpret_cast<const uint4*>(vr + (x >> 3) * kAtom + (x & 7) * 16);
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                odd |= (w[k] & 0x7F80u) == 0x7F80u || (w[k] & 0x7F800000u) == 0x7F800000u;
                        }
                        clear = odd;
                    }
                    if (drafts) {
                        const unsigned bits = __ballot_sync(0xffffffffu, clear && j < keys);
                        if (lane == 0) odd_drafts[q] = bits;
                    }
                    if (clear) {
#pragma unroll
                        for (int x = 0; x < S::kAtoms * 8; ++x)
                            *reinterpret_cast<uint4*>(vr + (x >> 3) * kAtom + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
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
            // a segment that is its whole group (both epilogue groups share it where KS = 2) is finished here
            const bool whole = sg.tile0 == 0 && sg.tile1 == sg.s.nt;
            if (KS == 2 ? both_groups_or(!alive) : group_or(bar, !alive)) break;  // who shares barriers leaves together
            tc_fence_after();
            // drafts whose V is not finite were left out of O: their P is still in its buffer, row by row
            if (sg.tile1 == sg.s.nt && (KS == 1 || ((sg.tile1 - 1 - sg.tile0) & 1) == nb) &&
                (odd_drafts[0] | odd_drafts[1] | odd_drafts[2] | odd_drafts[3])) {
#pragma unroll 1
                for (int r = 0; r < nr; ++r) {
                    float s = 0.f;
                    for (int x = 0; x < sg.s.n; ++x) {
                        if ((D == 64 && q >= 2) || !(odd_drafts[x >> 5] >> (x & 31) & 1)) continue;
                        if (!(rows_that_see(a, row0, sg.s.n, x, sg.r0 + base + r, 1) & 1)) continue;
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
                constexpr int kN = RB < 32 ? RB : 32;
                const auto plus = [](float x, float y) { return x + y; };
#pragma unroll
                for (int r = 0; r < RB; r += kN) {
                    float v[kN];
#pragma unroll
                    for (int k = 0; k < kN; k += 2) {
                        v[k] = l[(r + k) / 2].x;
                        v[k + 1] = l[(r + k) / 2].y;
                    }
                    const float x = reduce_scatter<kN>(v, lane, plus);
                    if (RB < 64) {
                        if (lane < kN) row_w[q * RB + r + lane] = x;
                    } else {
                        l[r / 2].x = x;
                    }
                }
            }
            if (RB < 64) {
                group_sync(bar);
                if (j < RB) row_f[j] = (row_w[j] + row_w[RB + j]) + (row_w[2 * RB + j] + row_w[3 * RB + j]);
            } else {  // row_w is the P buffer, which may be wanted yet: warp after warp
#pragma unroll 1
                for (int w = 0; w < 4; ++w) {
                    if (q == w)
#pragma unroll
                        for (int r = 0; r < RB; r += 32) row_f[r + lane] = (w > 0 ? row_f[r + lane] : 0.f) + l[r / 2].x;
                    group_sync(bar);
                }
            }
            if (!whole) {
                const int64_t part = ((int64_t)(cta + sg.group) * KS + (KS == 2 ? nb : 0)) * a.RB + base;
                group_sync(bar);
                if (j < nr) a.part_ml[part + j] = make_float2(row_m[j], row_f[j]);
#pragma unroll 1
                for (int r = 0; r < RB; r += kCols) {
                    if (r >= nr) break;
                    float hi[kCols], lo[kCols];
                    tmem_ld_cols<kCols>(t_o + r, hi);
                    tmem_ld_cols<kCols>(t_o + RB + r, lo);
                    tmem_wait_ld();
                    tie<kCols>(hi);
                    tie<kCols>(lo);
                    if (D == 128 || q < 2) {
#pragma unroll
                        for (int k = 0; k < kCols; ++k) {
                            if (r + k >= nr) break;
                            a.part_o[(part + r + k) * D + j] = live ? hi[k] + lo[k] : 0.f;
                        }
                    }
                }
            } else {
                // what the groups' O count in o (a group without a key counts 0)
                float* row_a = KS == 2 ? row_n + RB : row_f;
                float* row_b = row_a + RB;
                if (KS == 2) both_groups_or(false);
                else group_sync(bar);
                tc_fence_after();
                if (j < RB) {
                    float M = row_m[j], L = row_f[j], fa = 1.f, fb = 0.f;
                    if (KS == 2) {
                        const float* g0 = reinterpret_cast<const float*>(sm + S::kRowOff);
                        const float ma = g0[j], mb = g0[S::kRowArrays * RB + j];
                        M = fmaxf(ma, mb);
                        fa = ma == -INFINITY ? 0.f : ex2(ma - M);
                        fb = mb == -INFINITY ? 0.f : ex2(mb - M);
                        // NaN stays where a group has no maximum either
                        L = (fa != 0.f ? fa * g0[RB + j] : M == -INFINITY ? g0[RB + j] : 0.f) +
                            (fb != 0.f ? fb * g0[S::kRowArrays * RB + RB + j] : M == -INFINITY ? g0[S::kRowArrays * RB + RB + j] : 0.f);
                        if (L != L) fa = fb = 1.f;
                    }
                    const bool none = M == -INFINITY && L == 0.f;
                    const float inv = none ? 0.f : 1.f / L;
                    if ((KS == 1 || nb == 0) && j < nr) {
                        const int rr = sg.r0 + base + j, h = sg.g * a.rep + rr % a.rep;
                        const int64_t row = row0 + rr / a.rep;
                        if (a.lse != nullptr) a.lse[(int64_t)h * a.n_rows + row] = L == 0.f ? -INFINITY : fmaf(M, kLn2, logf(L));
                        if (a.factor != nullptr) a.factor[row * a.Hq + h] = weight_factor(a, make_float2(M, L), row);
                    }
                    row_a[j] = fa * inv;
                    if (KS == 2) row_b[j] = fb * inv;
                }
                group_sync(bar);
                // o of half the rows (KS = 2), or of the group's: lane = column
                constexpr int kMine = KS == 2 ? RB / 2 : RB, kStep = kMine < 16 ? (kMine < 8 ? 4 : 8) : 16;
                const uint32_t t_a = KS == 2 ? tmem + lane_off + (uint32_t)S::kOCol : t_o;
#pragma unroll 1
                for (int r = KS == 2 ? nb * kMine : 0, end = r + kMine; r < end; r += kStep) {
                    if (r >= nr) break;
                    float hi[kStep], lo[kStep], hb[kStep], lb[kStep];
                    tmem_ld_cols<kStep>(t_a + r, hi);
                    tmem_ld_cols<kStep>(t_a + RB + r, lo);
                    if (KS == 2) {
                        tmem_ld_cols<kStep>(t_a + 2 * RB + r, hb);
                        tmem_ld_cols<kStep>(t_a + 3 * RB + r, lb);
                    }
                    tmem_wait_ld();
                    tie<kStep>(hi);
                    tie<kStep>(lo);
                    if (KS == 2) {
                        tie<kStep>(hb);
                        tie<kStep>(lb);
                    }
                    if (D == 128 || q < 2) {
#pragma unroll
                        for (int k = 0; k < kStep; ++k) {
                            if (r + k >= nr) break;
                            const float wa = row_a[r + k], wb = KS == 2 ? row_b[r + k] : 0.f;
                            float o = wa != 0.f && (KS == 2 || live) ? (hi[k] + lo[k]) * wa : 0.f;
                            if (KS == 2 && wb != 0.f) o = fmaf(hb[k] + lb[k], wb, o);
                            const int rr = sg.r0 + base + r + k, h = sg.g * a.rep + rr % a.rep;
                            reinterpret_cast<__nv_bfloat16*>(a.out)[((row0 + rr / a.rep) * a.Hq + h) * D + j] = __float2bfloat16_rn(o);
                        }
                    }
                }
                tc_fence_before();
                if (KS == 2) both_groups_or(false);  // O is read: the next segment's may begin
            }
            tc_fence_before();
            group_sync(bar);  // row_w, row_m and P are free for the next segment
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && *abort_flag) {
        // a CTA that gave up: the last copy into every slot of the ring lands before it exits (all others
        // have been waited for by the issuers)
        const int n = 2 * max(issued_tiles[0], issued_tiles[1]);
        uint32_t seen = 0;
        for (int e = n - 1; e >= 0 && e >= n - 2 * S::kStages; --e) {
            const int slot = e % S::kStages;
            if (e / 2 >= issued_tiles[e & 1] || (seen >> slot & 1)) continue;
            seen |= 1u << slot;
            drain_wait(&full[slot], (e / S::kStages) & 1, a.status);
        }
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmem));
    }
}

// The weights with the scores formed again (see cache_attn.cu): S^T = K Q^T tile by tile with every
// row of the (b, KV head) resident, w_j = sum_r c_r 2^(S_jr c - M_r) / L_r, a thread a key.  A CTA takes
// an equal run of the call's (b, KV head, tile); the blocks of 64 rows of a tile go to the two groups
// in turn, whose sums are added in their order.  Rows beyond kWRows take another pass over the run,
// by the same threads.  Bound by K's bytes up to some 170 rows a KV head, then by ex2 (16 a clock).
constexpr int kWRows = 448, kWBlock = 64, kWMinStages = 3, kWMaxStages = 6, kWBufs = 4;
template <int D>
struct WShape {
    static constexpr int kAtoms = D / 64;
    static constexpr int kTileBytes = kAtoms * kAtom;
    static constexpr int kBlockBytes = kAtoms * kWBlock * 128;  // Q of one block of rows
    // from a 1024-aligned base: barriers, factors and sums first, then Q blocks and as many K tiles as fit
    static constexpr int kBars = 2 * kWMaxStages + 1 + 4 * kWBufs + 1;
    static constexpr int kMiscOff = kBars * 8;          // tmem address, abort flag
    static constexpr int kRedOff = 256;                 // [2][128] the second group's sums
    static constexpr int kFOff = kRedOff + 2 * 128 * 4; // [kWRows] factors
    static constexpr int kQOff = (kFOff + kWRows * 8 + 1023) / 1024 * 1024;
    static_assert(kMiscOff + 8 <= kRedOff, "barriers");
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
                     "r"(2 * kWBufs * kWBlock));
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
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the factors are complete

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
            constexpr uint32_t kId = idesc_bf16(kCacheTile, kWBlock);
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
                        for (int k = 0; k < blocks; ++k) {
                            const int gr = k & 1;
                            const uint32_t n = steps[gr]++, buf = n % kWBufs, use = n / kWBufs;
                            if (use >= 1 && !wait(&s_empty[gr * kWBufs + buf], (use - 1) & 1)) break;
                            tc_fence_after();
                            issued = true;
                            const uint32_t qa = smem_u32(sm + S::kQOff + k * S::kBlockBytes);
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk)
                                mma_bf16<kId>(tmem + (gr * kWBufs + buf) * kWBlock,
                                              sw128_desc(ka + (kk >> 2) * kAtom + (kk & 3) * 32),
                                              sw128_desc(qa + (kk >> 2) * kWBlock * 128 + (kk & 3) * 32), kk > 0 ? 1u : 0u);
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
        float2* fs = reinterpret_cast<float2*>(sm + S::kFOff);
        float* red = reinterpret_cast<float*>(sm + S::kRedOff);
        uint32_t step = 0, parity = 0;
        bool alive = true;
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
                    const uint32_t at = smem_u32(sm + S::kQOff) + (r / kWBlock) * S::kBlockBytes + (ch >> 3) * kWBlock * 128 +
                                        (r % kWBlock) * 128 + (((ch & 7) ^ (r & 7)) << 4);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(r < nr ? 16 : 0)
                                 : "memory");
                }
                for (int r = tid; r < blocks * kWBlock; r += 256)
                    fs[r] = r < nr ? a.factor[(row0 + (r0 + r) / a.rep) * a.Hq + w.g * a.rep + (r0 + r) % a.rep]
                                   : make_float2(0.f, 0.f);
                asm volatile("cp.async.wait_all;" ::: "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                both_groups_or(false);  // the factors are everyone's
                if (lane == 0) mbar_arrive(q_full);
                for (int tile = w.tile0; tile < w.tile1; ++tile, parity ^= 1) {
                    const bool drafts = tile == w.s.nt - 1;
                    const int keys = tile_keys(a, w.s, tile);
                    float* to = nullptr;
                    float had = 0.f;
                    if (gr == 0 && j < keys) {  // early: its latency passes under the sums
                        if (drafts) {
                            to = a.w_new + (row0 + j) * a.c.Hkv + w.g;
                            if (r0 > 0) had = *to;
                        } else {
                            const int slot = tile * kCacheTile + j;
                            const int64_t page = a.c.page_of(w.b, slot, a.status);
                            if (page >= 0) {
                                to = a.c.weight + a.c.meta(page, slot, w.g);
                                had = *to;
                            }
                        }
                    }
                    float sum[2] = {0.f, 0.f};
                    for (int k = gr; k < blocks; k += 2, ++step) {
                        const uint32_t buf = step % kWBufs;
                        if (alive)
                            alive = warp_wait(&s_full[gr * kWBufs + buf], (step / kWBufs) & 1, abort_flag, a.status, a.wait_cycles);
                        tc_fence_after();
                        const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16) + (gr * kWBufs + buf) * kWBlock;
                        const int cols = min(kWBlock, nr - k * kWBlock);
                        const uint64_t seen = drafts ? rows_that_see(a, row0, keys, j, r0 + k * kWBlock, cols) : ~0ull;
                        float z[kWBlock];
#pragma unroll
                        for (int c = 0; c < kWBlock; c += 16) tmem_ld16(ta + c, z + c);
                        tmem_wait_ld();
                        tie<kWBlock>(z);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&s_empty[gr * kWBufs + buf]);
                        const float4* f4 = reinterpret_cast<const float4*>(fs + k * kWBlock);
#pragma unroll
                        for (int c = 0; c < kWBlock; c += 16) {
                            if (c >= cols) break;
#pragma unroll
                            for (int i = c; i < c + 16; i += 2) {  // columns past the rows have a factor of 0
                                const float4 f = f4[i / 2];
                                const float e0 = ex2(fmaf(z[i], a.scale_log2, f.x)), e1 = ex2(fmaf(z[i + 1], a.scale_log2, f.z));
                                sum[0] = f.y != 0.f && (seen >> i & 1) ? fmaf(e0, f.y, sum[0]) : sum[0];
                                sum[1] = f.w != 0.f && (seen >> i & 2) ? fmaf(e1, f.w, sum[1]) : sum[1];
                            }
                        }
                    }
                    const float mine = sum[0] + sum[1];
                    if (gr == 1) red[parity * 128 + j] = mine;
                    if (both_groups_or(!alive)) {
                        alive = false;
                        break;
                    }
                    if (to != nullptr) *to = had + (mine + red[parity * 128 + j]);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kWBufs * kWBlock));
    }
}

// Pages as (d, slot, KV head, page); a box is 64 values of box_rows slots of one head.
estp_status pages_map(CUtensorMap* m, const CacheView& c, const void* base, const void* other, int box_rows) {
    auto fn = tensor_map_encoder();
    if (!fn) return fail(ESTP_ERR_CUDA, "cuTensorMapEncodeTiled unavailable");
    const bool none = c.n_pages == 0;  // no page can be read: a map of the right form over another array
    cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)1 << c.shift, (cuuint64_t)c.Hkv, none ? 1 : (cuuint64_t)c.n_pages};
    cuuint64_t strides[3] = {(cuuint64_t)c.slot_stride, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride};
    cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, es[4] = {1, 1, 1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(none ? other : base), dims, strides, box,
                          es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ESTP_OK : fail(ESTP_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

// New rows as (d, KV head, row); a box is 64 values of box_rows rows of one head.
estp_status rows_map(CUtensorMap* m, const CacheAttnArgs& a, const void* base, int box_rows) {
    auto fn = tensor_map_encoder();
    if (!fn) return fail(ESTP_ERR_CUDA, "cuTensorMapEncodeTiled unavailable");
    const bool none = base == nullptr;  // never read
    cuuint64_t dims[3] = {(cuuint64_t)a.c.d, (cuuint64_t)(none ? 1 : a.c.Hkv), (cuuint64_t)a.n_rows};
    cuuint64_t strides[2] = {(cuuint64_t)a.c.d * 2, (cuuint64_t)(none ? a.ldq : a.ldn)};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows}, es[3] = {1, 1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(none ? (const void*)a.Q : base), dims,
                          strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ESTP_OK : fail(ESTP_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

template <int D, int RB, int KS>
estp_status launch(estp_ctx* ctx, const TcMaps& tm, const CacheAttnArgs& a, int box_rows, int new_rows, cudaStream_t st) {
    using S = Shape<D, RB, KS>;
    constexpr int kBit = 2 + (D == 128 ? 8 : 0) + (RB == 8 ? 0 : RB == 16 ? 1 : RB == 32 ? 2 : KS == 2 ? 3 : 4);
    cudaError_t e = set_smem(ctx, kBit, cache_fwd_tc_kernel<D, RB, KS>, S::kSmem);
    if (e != cudaSuccess) return cuda_fail(e, "cache attention smem attribute");
    cache_fwd_tc_kernel<D, RB, KS><<<(unsigned)a.G, S::kThreads, S::kSmem, st>>>(tm, a, box_rows, new_rows);
    e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache attention launch");
}

template <int D>
estp_status launch_rows(estp_ctx* ctx, const TcMaps& tm, const CacheAttnArgs& a, int box_rows, int new_rows, cudaStream_t st) {
    switch (a.RB) {
        case 8: return launch<D, 8, 2>(ctx, tm, a, box_rows, new_rows, st);
        case 16: return launch<D, 16, 2>(ctx, tm, a, box_rows, new_rows, st);
        case 32: return launch<D, 32, 2>(ctx, tm, a, box_rows, new_rows, st);
        case 64: return launch<D, 64, 2>(ctx, tm, a, box_rows, new_rows, st);
        default: return launch<D, 64, 1>(ctx, tm, a, box_rows, new_rows, st);
    }
}

}  // namespace

void cache_tc_shape(int rows, int* RB, int* KS) {
    *RB = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    *KS = rows <= 64 ? 2 : 1;
}

static estp_status make_maps(const CacheAttnArgs& a, TcMaps* tm, int* box_rows, int* new_rows) {
    const int page = 1 << a.c.shift;
    *box_rows = page < kCacheTile ? page : kCacheTile;
    *new_rows = (a.max_rows + 7) / 8 * 8;
    estp_status s = pages_map(&tm->k, a.c, a.c.k, a.Q, *box_rows);
    if (s == ESTP_OK) s = pages_map(&tm->v, a.c, a.c.v, a.Q, *box_rows);
    if (s == ESTP_OK) s = rows_map(&tm->kn, a, a.kn, *new_rows);
    if (s == ESTP_OK) s = rows_map(&tm->vn, a, a.vn, *new_rows);
    return s;
}

estp_status launch_cache_fwd_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st) {
    TcMaps tm;
    int box_rows, new_rows;
    const estp_status s = make_maps(a, &tm, &box_rows, &new_rows);
    if (s != ESTP_OK) return s;
    return a.c.d == 128 ? launch_rows<128>(ctx, tm, a, box_rows, new_rows, st) : launch_rows<64>(ctx, tm, a, box_rows, new_rows, st);
}

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
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctx->num_sms);
    cfg.blockDim = dim3(WShape<128>::kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, tm, a, box_rows, new_rows, blocks, stages);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache weight launch");
}

}  // namespace estp
