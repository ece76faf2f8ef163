// What the tensor-core kernels of the cache share: TMEM and TMA helpers, the walk over a CTA's units,
// the copies of a tile of keys and the tensor maps.
#pragma once

#include "cache.cuh"
#include "tcgen05.cuh"

namespace estp {

constexpr int kAtom = kCacheTile * 128;  // 128 keys x 64 bf16

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

// The issue of a product is a thread's own instructions: descriptors are formed once and stepped by adding
// (the address field counts 16 bytes and does not overflow), and whole tiles are unrolled.  Formed anew
// and looped over, an MMA took 140 clocks to issue where the pipe needs 64.

// D (TMEM) = K Q^T or Q K^T: both K-major, rows of A and B 128 bytes, second 64 columns lead_a, lead_b on
template <uint32_t kIdesc, int D>
__device__ __forceinline__ void product_k_major(uint32_t d_tmem, uint32_t a, uint32_t lead_a, uint32_t b, uint32_t lead_b) {
    const uint64_t ad = sw128_desc(a), bd = sw128_desc(b);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
        mma_bf16<kIdesc>(d_tmem, ad + (kk >> 2) * (lead_a >> 4) + (kk & 3) * 2, bd + (kk >> 2) * (lead_b >> 4) + (kk & 3) * 2,
                         kk > 0 ? 1u : 0u);
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
    template <int kRB = 0>
    __device__ __forceinline__ bool next(const CacheAttnArgs& a, Segment& o) {
        while (u < u1) {
            o.s = seq_shape<kRB>(a, at.b);
            if (u >= at.unit0 + o.s.units(a.c.Hkv)) {
                at.pass(o.s, a.c.Hkv);
                continue;
            }
            const Span x = span_of<kRB>(a, o.s, u - at.unit0, u1 - u);
            u += x.units;
            if (x.tile0 >= x.tile1) continue;
            o.tile0 = x.tile0;
            o.tile1 = x.tile1;
            o.b = at.b;
            o.g = x.g;
            o.r0 = x.k * a.RB;
            o.nr = min(a.RB, o.s.n * a.rep - o.r0);
            o.group = at.group0 + x.g * o.s.nrb + x.k;
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

// A key's V row in shared memory (128-byte swizzled atoms): whether a value of it is not finite; zeros.
template <int D>
__device__ __forceinline__ bool row_not_finite(const uint8_t* row) {
    bool odd = false;
#pragma unroll 2
    for (int x = 0; x < D / 8; ++x) {
        const uint4 v = *reinterpret_cast<const uint4*>(row + (x >> 3) * kAtom + (x & 7) * 16);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) odd |= (w[k] & 0x7F80u) == 0x7F80u || (w[k] & 0x7F800000u) == 0x7F800000u;
    }
    return odd;
}
template <int D>
__device__ __forceinline__ void clear_row(uint8_t* row) {
#pragma unroll 1
    for (int x = 0; x < D / 8; ++x) *reinterpret_cast<uint4*>(row + (x >> 3) * kAtom + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
}

// The rings of K and V tiles.  Each has its own slots and its own producer warp: a slot's barriers are
// followed by parity, which holds only if one warp issues all of the slot's copies in order (shared by two,
// a warp that was a phase ahead of the other would take a phase two back for its own).
struct Ring {
    uint64_t *full, *empty;
    uint8_t* tiles;
    int n, tile_bytes;
    __device__ __forceinline__ int slot(uint32_t t) const { return (int)(t % n); }
    __device__ __forceinline__ uint32_t parity(uint32_t t) const { return (t / n) & 1; }
    __device__ __forceinline__ uint8_t* tile(uint32_t t) const { return tiles + slot(t) * tile_bytes; }
    __device__ __forceinline__ uint64_t* filled(uint32_t t) const { return &full[slot(t)]; }
    __device__ __forceinline__ uint64_t* freed(uint32_t t) const { return &empty[slot(t)]; }
    // a CTA that gave up: the last copy into every slot lands before it exits (others have been waited for)
    __device__ __forceinline__ void drain(int issued, int* status) const {
        for (int t = issued - 1; t >= 0 && t >= issued - n; --t) drain_wait(filled(t), parity(t), status);
    }
};

// Pages as (d, slot, KV head, page); a box is 64 values of box_rows slots of one head.
inline estp_status pages_map(CUtensorMap* m, const CacheView& c, const void* base, const void* other, int box_rows) {
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
inline estp_status rows_map(CUtensorMap* m, const CacheAttnArgs& a, const void* base, int box_rows) {
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

inline estp_status make_maps(const CacheAttnArgs& a, TcMaps* tm, int* box_rows, int* new_rows) {
    const int page = 1 << a.c.shift;
    *box_rows = page < kCacheTile ? page : kCacheTile;
    *new_rows = (a.max_rows + 7) / 8 * 8;
    estp_status s = pages_map(&tm->k, a.c, a.c.k, a.Q, *box_rows);
    if (s == ESTP_OK) s = pages_map(&tm->v, a.c, a.c.v, a.Q, *box_rows);
    if (s == ESTP_OK) s = rows_map(&tm->kn, a, a.kn, *new_rows);
    if (s == ESTP_OK) s = rows_map(&tm->vn, a, a.vn, *new_rows);
    return s;
}


}  // namespace estp
