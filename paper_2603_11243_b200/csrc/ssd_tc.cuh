// Wrappers of the sm_100a instructions that the cache's kernels are built from: tensor-map copies,
// 5th-generation tensor-core products with their accumulators in tensor memory, and the layouts
// both agree on.
//
// Layout of every operand tile in shared memory: rows of 64 sixteen-bit values (128 bytes), the
// 16-byte units of a row XORed with the row's number modulo 8 (the 128-byte swizzle), 1,024-byte
// aligned.  A head of D values is D / 64 such blocks one behind the other, each of 128 rows.  Read
// along a row it is a K-major operand (queries and keys in the scores); read along the rows it is
// the MN-major one (values in the second product).
#pragma once

#include <cuda.h>
#include <float.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ssd_common.cuh"

namespace ssd {
namespace tc {

constexpr int kTile = 128;                       // rows of a tile: queries, and keys
constexpr int kBlockBytes = kTile * 128;         // 64 columns of a tile

// ---- tensor-map copies -------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}

// ---- tensor memory -------------------------------------------------------------------------------
// Taken before griddepcontrol.launch_dependents: once a successor may start, everyone of this grid
// already has its columns, so neither waits for the other's.
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: lane i of the warp gets row i.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float *r) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
          "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]),
          "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]),
          "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float *r) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
          "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *u) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
          "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(addr)
        : "memory");
}

// ---- products --------------------------------------------------------------------------------------
// Shared-memory descriptor of an operand at `addr`, 128-byte swizzle: bits 0-13 address / 16,
// 16-29 leading offset / 16, 32-45 stride offset / 16, 46-47 the descriptor's version, 61-63 swizzle.
// K-major: 8 rows lie 1,024 bytes apart (the leading offset is not looked at).  MN-major: 8 rows of
// the K axis lie 1,024 bytes apart, blocks of 64 columns kBlockBytes.
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(kBlockBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor: fp32 accumulators, both operands of one 16-bit type, M = 128.
template <typename T> struct Format;
template <> struct Format<__half> { static constexpr uint32_t kCode = 0, kExponent = 0x7c00; };
template <> struct Format<__nv_bfloat16> { static constexpr uint32_t kCode = 1, kExponent = 0x7f80; };
template <typename T> __device__ __forceinline__ uint32_t instruction(uint32_t n, bool b_mn_major) {
    return 1u << 4 | Format<T>::kCode << 7 | Format<T>::kCode << 10 | (b_mn_major ? 1u << 16 : 0u) | (n >> 3) << 17 |
           (uint32_t)(kTile >> 4) << 24;
}
// One thread of a converged warp.  Products are issued under this and with operands that are the same in
// every lane as far as the compiler can see: under `lane == 0` each operand of each of them is moved to a uniform
// register first, and eight products of 64 clocks took 1,000 to issue.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// the value of lane 0, in every lane
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
// d (+)= a . b; a and b in shared memory
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// d (+)= a . b; a in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// arrives on `bar` once every product this thread has issued so far is complete
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- small arithmetic -----------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// x -> cap tanh(scale x / cap) of N scores a thread.  Scores well below the cap, as nearly all are, take an odd
// polynomial (tanh(y) / y in y^2 on |y| <= 1/2, coefficients by Remez's exchange: within 2.8e-8 of it, at 1/2): eight
// packed operations for two scores and none on the special-function unit, which the softmax needs.  Where a
// score of the warp is larger, y >= 1/2 goes through 1 - 2 / (1 + e^2y): its error, 1e-7, is then relative to
// at least 0.46.
// `counts`: whether the thread's scores are anybody's (what lies in other rows must not send a warp the long way).
template <int N> __device__ __forceinline__ void cap_scores(float *x, float scale, float cap, bool counts) {
    const float r = fminf(scale / cap, FLT_MAX);         // of a cap of no size: a score of 0 stays 0, others become the cap
    constexpr float c1 = -0.33333069394019127f, c2 = 0.13324779317551644f, c3 = -0.05298607528769192f, c4 = 0.01713500662684319f;
    float top[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) top[k] = fmaxf(fmaxf(top[k], fabsf(x[i + k])), fabsf(x[i + 4 + k]));      // NaN stays NaN either way
    const bool all_small = __all_sync(0xffffffffu, !counts || fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * r <= 0.5f);
    auto poly = [&](float2 v) {
        const float2 y = fmul2(v, make_float2(r, r)), t = fmul2(y, y);
        float2 q = ffma2(make_float2(c4, c4), t, make_float2(c3, c3));
        q = ffma2(q, t, make_float2(c2, c2));
        q = ffma2(q, t, make_float2(c1, c1));
        q = ffma2(q, t, make_float2(1.f, 1.f));
        return fmul2(q, fmul2(y, make_float2(cap, cap)));
    };
    if (all_small) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 q = poly(make_float2(x[i], x[i + 1]));
            x[i] = q.x;
            x[i + 1] = q.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 q = poly(make_float2(x[i], x[i + 1]));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float y = x[i + k] * r;
                const float big = cap - __fdividef(2.f * cap, 1.f + ex2(2.f * kLog2e * y));
                x[i + k] = fabsf(y) <= 0.5f ? (k ? q.y : q.x) : big;
            }
        }
    }
}
// The cap that the kernels take.  Where scale / cap lies below fp32's normal numbers it would lose digits, and the cap
// changes nothing: cap tanh(s / cap) is s but for (s / cap)^2 / 3 of it, 5e-9 for a product of query and key of 1e34.
inline float cap_in_range(float scale, float cap) { return cap > 0.f && scale / cap < FLT_MIN ? 0.f : cap; }
// where the 16-byte unit `unit` of row `row` of a tile lies
__device__ __forceinline__ uint32_t unit_at(uint32_t tile, int row, int unit) {
    return tile + (unit >> 3) * kBlockBytes + row * 128 + (((unit & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ void named_sync(int id, int threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// ---- the paged cache's tiles ------------------------------------------------------------------------
// A tile is up to 128 consecutive slots that end within `pages` whole pages (pages of up to 64 slots,
// a multiple of 8: as many as fit; other pages of up to 128: one) or within one page (larger pages).
// The swizzle's pattern repeats every 8 rows, so a copy lands on a multiple of 8.  A page of up to 64 slots that is none
// is a tile of its own, which costs what a full one does: trees of 5 to 32 nodes on 64 caches of 500 to 3,000 slots take
// 113 us with pages of 16, 166 of 60, 356 of 20, 1,574 of 4 and 6,145 of one slot.
struct Paging {
    int page;          // slots of a page
    int pages;         // pages of a tile; 0: tiles within a page
    int per_page;      // tiles of a page where pages == 0
    int box;           // slots that one copy brings
};
inline Paging paging(int page) {
    Paging p{};
    p.page = page;
    if (page <= kTile) {
        p.pages = page <= 64 && page % 8 == 0 ? kTile / page : 1;
        p.box = page;
    } else {
        p.per_page = (page + kTile - 1) / kTile;
        p.box = 64;
    }
    return p;
}
constexpr int64_t kMostSlots = INT32_MAX - 256;      // of an utterance, so that rounding up to tiles stays in 32 bits
struct TileAt {
    int page, slot, valid;    // first page (of the utterance's table), first slot in it, slots that count
};
__host__ __device__ inline int paged_tiles(const Paging &p, int len) {
    if (p.pages) return (len + p.pages * p.page - 1) / (p.pages * p.page);
    const int whole = len / p.page, rest = len - whole * p.page;
    return whole * p.per_page + (rest + kTile - 1) / kTile;
}
__host__ __device__ inline TileAt paged_tile(const Paging &p, int len, int t) {
    TileAt a;
    if (p.pages) {
        a.page = t * p.pages;
        a.slot = 0;
        const int left = len - a.page * p.page, most = p.pages * p.page;
        a.valid = left < most ? left : most;
    } else {
        a.page = t / p.per_page;
        a.slot = (t - a.page * p.per_page) * kTile;
        const int in_page = p.page - a.slot, left = len - a.page * p.page - a.slot;
        a.valid = in_page < kTile ? in_page : kTile;
        if (left < a.valid) a.valid = left;
    }
    return a;
}

}  // namespace tc

// ---- host: tensor maps ---------------------------------------------------------------------------
// dims[0] is the innermost axis (contiguous); strides[i] is axis i + 1's, in bytes.  False: the
// driver refused (or there is none); record_cuda_error has been called.
bool encode_map(CUtensorMap *map, ssd_dtype dtype, const void *base, int rank, const uint64_t *dims,
                const uint64_t *strides, const uint32_t *box);
bool encode_rows(CUtensorMap *map, ssd_dtype dtype, const ssd_heads &x, int D, int64_t M, int box_heads, int box_rows);
bool encode_cache(CUtensorMap *map, const ssd_kv_cache &c, const void *data, int box);

}  // namespace ssd
