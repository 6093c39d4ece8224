// Attention for draft trees over a paged key/value cache (ssd_tree_attention).
//
// Every node of an utterance's tree attends to the utterance's cache and to its own line of
// descent: out_i = sum_j softmax_j(s_ij) v_j with s_ij = scale q_i.k_j, or cap tanh(scale q_i.k_j / cap).
// The query heads that share a kv head are rows of one product: a tile is 128 / G nodes by G heads, its
// keys come 128 at a time, and the softmax is carried as a running maximum and sum per row.
//
// One CTA of ten warps works on one kv head and up to two tiles of queries (one pass over the keys
// serves both) or, where the rows fill one tile or less, on one tile, whose key tiles then alternate
// between two accumulators.  Either way there are two streams of (scores -> softmax -> product), so the
// tensor cores work on one while the other's exponentials are taken: warps 0-3 and 4-7 hold one row a
// thread, warps 8 and 10 issue the copies, warp 9 the products.  Scores and accumulators live in tensor
// memory; probabilities go back there in 16 bits, over the scores they came from, and are the first
// operand of the second product.  Few rows and a long cache: the key tiles are split over a cluster
// of CTAs, whose partial results meet in shared memory, so a call is one launch and needs no scratch.
#include <math.h>

#include "ssd_tc.cuh"

namespace ssd {
namespace {

using namespace tc;

constexpr int kWarps = 12;                // 8 of softmax, 2 of copies, 1 of products, and one that fills their group
constexpr int kParents = 256;            // parents kept in shared memory; more are read from global
constexpr int kTreeBox = 16;             // nodes that one copy brings
constexpr int kMaxSplit = 8;

struct alignas(64) AttnParams {
    CUtensorMap q, tree_k, tree_v, cache_k, cache_v;
    const int32_t *table, *len, *parent;
    const int64_t *off;
    const void *tree_v_at;               // the same values as tree_v's
    int64_t tree_row, tree_head;
    void *out;
    int64_t out_row, out_head;
    float *lse;
    uint32_t *status;
    int64_t table_stride, M;
    int B, Hq, Hkv, G, npt, q_items, max_nodes, n_pages, max_pages, split;
    Paging paging;
    float scale, cap;
};

template <int D> struct Shape {
    static constexpr int kBlocks = D / 64;
    static constexpr int kSlotBytes = kBlocks * kBlockBytes;      // a tile of keys or of values
    static constexpr int kSlots = D == 128 ? 5 : 8;
    static constexpr int kRing = 2 * kSlotBytes;                  // behind the two tiles of queries
    static constexpr int kMisc = kRing + kSlots * kSlotBytes;
    static constexpr int kBars = kMisc;                           // q, full[], empty[], scores[2], probs[2], sums[2]
    static constexpr int kNumBars = 1 + 2 * kSlots + 6;
    static constexpr int kWords = kBars + kNumBars * 8;           // tmem address, failed, bad value seen
    static constexpr int kMl = (kWords + 16 + 15) / 16 * 16;      // [2][128] running maximum and sum
    static constexpr int kParent = kMl + 2 * kTile * 8;
    static constexpr int kBytes = kParent + kParents * 2;
    static constexpr size_t kDynamic = kBytes;
    static constexpr int kO = 256;                                // tensor memory: scores at 0 and 128, sums here
};
static_assert(Shape<128>::kDynamic <= 232448, "shared memory");
static_assert(2 * kTile * 128 * 4 <= Shape<128>::kSlots * Shape<128>::kSlotBytes, "partial results fit the ring");
static_assert(2 * kTile * 64 * 4 <= Shape<64>::kSlots * Shape<64>::kSlotBytes, "partial results fit the ring");

// What an item works on; the same in every thread.
struct Item {
    int64_t i0;          // first node of the utterance
    int b, h, n, len;
    int node0;           // first node of the item
    int pair;            // two tiles of queries
    int last;            // one past the last node that is a key
    int tree_tiles, begin, end;    // of the key tiles, this CTA's
    bool work;
};

__device__ __forceinline__ Item item_of(const AttnParams &p, int item, int rank) {
    Item it;
    const int qi = item % p.q_items;
    it.h = item / p.q_items % p.Hkv;
    it.b = item / p.q_items / p.Hkv;
    it.i0 = p.off[it.b];
    const int64_t i1 = p.off[it.b + 1];
    const bool ok = !(it.i0 < 0 || i1 < it.i0 || i1 > p.M || i1 - it.i0 > p.max_nodes);
    it.n = ok ? (int)(i1 - it.i0) : 0;
    const int64_t room = (int64_t)p.max_pages * p.paging.page;
    it.len = min(max(p.len[it.b], 0), (int)min(room, (int64_t)INT32_MAX));
    it.node0 = qi * 2 * p.npt;
    it.work = it.node0 < it.n;
    it.pair = it.n - it.node0 > p.npt;
    it.last = min(it.n, it.node0 + 2 * p.npt);
    it.tree_tiles = (it.last + kTile - 1) / kTile;
    const int total = it.tree_tiles + paged_tiles(p.paging, it.len);
    it.begin = (int)((int64_t)total * rank / p.split);
    it.end = (int)((int64_t)total * (rank + 1) / p.split);
    return it;
}
// The tree's own tiles come first, last nodes first: a thread walks its node's line upwards once.
__device__ __forceinline__ int tree_tile_start(const Item &it, int t) { return (it.tree_tiles - 1 - t) * kTile; }
__device__ __forceinline__ int tile_valid(const AttnParams &p, const Item &it, int t) {
    if (t < it.tree_tiles) return min(kTile, it.last - tree_tile_start(it, t));
    return paged_tile(p.paging, it.len, t - it.tree_tiles).valid;
}

// The utterance's status, by one warp of its first item.
__device__ __forceinline__ void report(const AttnParams &p, const Item &it, int item, int rank, bool failed, int lane) {
    if (it.h == 0 && item % p.q_items == 0 && rank == 0) {
        const int64_t i1 = p.off[it.b + 1];
        uint32_t bits = 0;
        if (it.i0 < 0 || i1 < it.i0 || i1 > p.M || i1 - it.i0 > p.max_nodes) bits |= SSD_UTT_BAD_OFFSETS;
        if (p.len[it.b] != it.len) bits |= SSD_UTT_BAD_CACHE;
        if (p.parent)
            for (int j = lane; j < it.n; j += 32) {
                const int up = p.parent[it.i0 + j];
                if (up < -1 || up >= j) bits |= SSD_UTT_BAD_PARENT;
            }
        const int pages = it.n > 0 ? (int)(((int64_t)it.len + p.paging.page - 1) / p.paging.page) : 0;
        for (int j = lane; j < pages; j += 32) {
            const int id = p.table[it.b * p.table_stride + j];
            if (id < 0 || id >= p.n_pages) bits |= SSD_UTT_BAD_CACHE;
        }
        bits = __reduce_or_sync(0xffffffffu, bits);
        if (lane == 0 && !failed) p.status[it.b] = bits;
    }
    if (failed && lane == 0) p.status[it.b] = SSD_UTT_INTERNAL;
}

__device__ __forceinline__ int up_from(const AttnParams &p, const Item &it, const int16_t *parents, int j) {
    if (!p.parent) return j - 1;
    if (j < kParents) return parents[j];
    const int up = p.parent[it.i0 + j];
    return up < -1 || up >= j ? -1 : up;
}

__device__ __forceinline__ bool not_finite16(uint32_t half_bits, uint32_t exponent) { return (half_bits & exponent) == exponent; }

// The product runs over whole groups of 16 keys, and 0 times NaN is NaN: values behind the last key
// are made zeros, and so are the tree's own values that are not finite (a node that does not see them
// must not get them; `seen` says that there are some, and those that do see them get them at the end).
template <typename T>
__device__ __forceinline__ void clean_values(uint32_t tile, int row, int valid, bool tree, int units, volatile uint32_t *seen) {
    if (row >= valid) {
        if (row < (valid + 15) / 16 * 16)
            for (int u = 0; u < units; ++u)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(unit_at(tile, row, u)), "r"(0) : "memory");
        return;
    }
    if (!tree) return;
    constexpr uint32_t e = Format<T>::kExponent;
    for (int u = 0; u < units; ++u) {
        uint32_t w[4];
        const uint32_t at = unit_at(tile, row, u);
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool lo = not_finite16(w[i], e), hi = not_finite16(w[i] >> 16, e);
            any |= lo || hi;
            w[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
        }
        if (any) {
            *seen = 1;
            __threadfence_block();
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        }
    }
}

// Probabilities are taken against a reference that may lag the running maximum, so that the sums are
// seldom scaled.  fp16 holds none below 6e-8: its probabilities are held times 2^10, with a lag of up
// to 2^4; bf16 has fp32's range, and the lag may be 2^8.
template <typename T> struct Lag {
    static constexpr float kLift = Format<T>::kCode == 0 ? 10.f : 0.f, kLag = Format<T>::kCode == 0 ? 4.f : 8.f;
};

template <typename T, int D, bool kCap>
__global__ void __launch_bounds__(kWarps * 32, 1) tree_attention(const __grid_constant__ AttnParams p) {
    using S = Shape<D>;
    extern __shared__ __align__(1024) uint8_t base[];          // the swizzle is a function of the address
    const uint32_t smem = smem_u32(base);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = blockIdx.x % p.split, item = blockIdx.x / p.split;

    const uint32_t q_full = smem + S::kBars;
    auto slot_full = [&](int i) { return smem + S::kBars + 8 + 8 * i; };
    auto slot_empty = [&](int i) { return smem + S::kBars + 8 + 8 * (S::kSlots + i); };
    const uint32_t more = smem + S::kBars + 8 + 16 * S::kSlots;
    auto scores_full = [&](int s) { return more + 8 * s; };
    auto probs_ready = [&](int s) { return more + 16 + 8 * s; };
    auto sums_full = [&](int s) { return more + 32 + 8 * s; };
    volatile uint32_t *const words = reinterpret_cast<volatile uint32_t *>(base + S::kWords);
    volatile uint32_t *const failed = words + 1, *const seen = words + 2;
    float2 *const ml = reinterpret_cast<float2 *>(base + S::kMl);
    int16_t *const parents = reinterpret_cast<int16_t *>(base + S::kParent);
    auto slot_at = [&](int pos) { return smem + S::kRing + (pos % S::kSlots) * S::kSlotBytes; };

    if (warp == 8) tmem_alloc(smem + S::kWords, 512);
    if (tid == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < S::kSlots; ++i) { mbar_init(slot_full(i), 1); mbar_init(slot_empty(i), 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(scores_full(s), 1);
            mbar_init(probs_ready(s), 4);
            mbar_init(sums_full(s), 1);
        }
        mbar_init_fence();
        words[1] = words[2] = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = words[0];
    pdl_wait();

    const Item it = item_of(p, item, rank);
    const int T_ = it.work ? it.end - it.begin : 0;                 // key tiles of this CTA
    const int units = it.pair ? 2 * T_ : T_;                        // (stream, tile) pairs, in the order of their products

    if (warp >= 8) {
      // of the 168 registers a thread is launched with, softmax threads get 224 and these keep 56
      asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
      if ((warp == 8 || warp == 10) && T_ > 0) {
        // ---- copies: queries and keys, and values, a warp each (it is the issue of many small copies that takes time) -----------------------------------------------------------------------------
        const int kv = warp == 10;
        if (!kv && lane == 0) {
            const int tiles = it.pair ? 2 : 1;
            mbar_arrive_expect_tx(q_full, tiles * S::kBlocks * p.G * p.npt * 128);
            for (int i = 0; i < tiles; ++i)
                for (int x = 0; x < S::kBlocks; ++x)
                    tma_load_3d(smem + i * S::kSlotBytes + x * kBlockBytes, &p.q, x * 64, it.h * p.G,
                                (int)it.i0 + it.node0 + i * p.npt, q_full);
        }
        const int32_t *const table = p.table + it.b * p.table_stride;
        const int page_count = p.paging.pages ? p.paging.pages : 1;
        auto page_id = [&](int t) {                                  // lane i: the tile's i-th page
            if (t < it.tree_tiles || t >= it.end || lane >= page_count) return 0;
            const TileAt a = paged_tile(p.paging, it.len, t - it.tree_tiles);
            if (a.page + lane >= p.max_pages) return p.n_pages;
            const int id = table[a.page + lane];
            return id < 0 || id >= p.n_pages ? p.n_pages : id;       // outside: the copy fills in zeros
        };
        int next = page_id(it.begin);
        bool ok = true;
        for (int t = it.begin; t < it.end && ok; ++t) {
            const int id = next;
            next = page_id(t + 1);
            const bool tree = t < it.tree_tiles;
            const int valid = tile_valid(p, it, t);
            const int box = tree ? kTreeBox : p.paging.box, copies = (valid + box - 1) / box;
            const int t0 = tree ? tree_tile_start(it, t) : 0;
            const int slot0 = tree ? 0 : paged_tile(p.paging, it.len, t - it.tree_tiles).slot;
            const int pos = 2 * (t - it.begin) + kv;
            if (pos >= S::kSlots) ok = mbar_wait_bounded(slot_empty(pos % S::kSlots), (pos / S::kSlots - 1) & 1);
            if (!ok) break;
            const uint32_t bar = slot_full(pos % S::kSlots);
            if (lane == 0) mbar_arrive_expect_tx(bar, copies * box * 128 * S::kBlocks);
            // a lane for every copy: of 64 columns and 8 rows at least, so 32 lanes are enough
            const int i = lane / S::kBlocks, x = lane % S::kBlocks;
            const int page = __shfl_sync(0xffffffffu, id, p.paging.pages ? i : 0);
            if (i < copies) {
                const uint32_t dst = slot_at(pos) + x * kBlockBytes + i * box * 128;
                if (tree)
                    tma_load_3d(dst, kv ? &p.tree_v : &p.tree_k, x * 64, it.h, (int)it.i0 + t0 + i * box, bar);
                else
                    tma_load_4d(dst, kv ? &p.cache_v : &p.cache_k, x * 64, it.h, p.paging.pages ? 0 : slot0 + i * box, page, bar);
            }
        }
        if (!ok) *failed = 1;
      } else if (warp == 9 && T_ > 0) {
        // ---- products ---------------------------------------------------------------------------
        bool ok = mbar_wait_bounded(q_full, 0);
        auto scores = [&](int u) {
            const int s = u & 1, tile = it.pair ? u >> 1 : u, pos = 2 * tile, valid = tile_valid(p, it, it.begin + tile);
            ok = ok && mbar_wait_bounded(slot_full(pos % S::kSlots), (pos / S::kSlots) & 1);
            if (!ok) return;
            tc_fence_after();
            if (lane == 0) {
                const uint32_t idesc = instruction<T>((valid + 15) / 16 * 16, false);
                const uint64_t a = operand(smem + (it.pair ? s : 0) * S::kSlotBytes), k = operand(slot_at(pos));
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const int at = (x >> 2) * (kBlockBytes >> 4) + (x & 3) * 2;       // 16 columns = 32 bytes of a block's rows
                    mma_ss(tmem + s * kTile, a + at, k + at, idesc, x > 0);
                }
                mma_commit(scores_full(s));
                if (!it.pair || s) mma_commit(slot_empty(pos % S::kSlots));
            }
            __syncwarp();
        };
        auto values = [&](int u) {
            const int s = u & 1, k = u >> 1, tile = it.pair ? k : u, pos = 2 * tile + 1, valid = tile_valid(p, it, it.begin + tile);
            ok = ok && mbar_wait_bounded(probs_ready(s), k & 1) &&
                 mbar_wait_bounded(slot_full(pos % S::kSlots), (pos / S::kSlots) & 1);
            if (!ok) return;
            tc_fence_after();
            if (lane == 0) {
                const uint32_t idesc = instruction<T>(D, true);
                const uint64_t v = operand(slot_at(pos));
                const int steps = (valid + 15) / 16;
                for (int x = 0; x < steps; ++x)                                       // 16 keys = 2,048 bytes of a block
                    mma_ts(tmem + S::kO + s * D, tmem + s * kTile + x * 8, v + x * (2048 >> 4), idesc, k > 0 || x > 0);
                if (!it.pair || s) mma_commit(slot_empty(pos % S::kSlots));
                if (u + 2 >= units) mma_commit(sums_full(s));
            }
            __syncwarp();
        };
        scores(0);
        if (units > 1) scores(1);
        for (int u = 0; u < units && ok; ++u) {
            values(u);
            if (u + 2 < units) scores(u + 2);
        }
        if (!ok) *failed = 1;
      }
      if (p.split > 1) { cluster_arrive(); cluster_wait(); cluster_arrive(); cluster_wait(); }
      named_sync(0, kWarps * 32);
      if (*failed) drain_after_error();
      if (warp == 8) {
        tc_fence_after();
        tmem_free(tmem, 512);
        report(p, it, item, rank, *failed != 0, lane);
      }
      return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    if (it.work) {
        // ---- softmax ------------------------------------------------------------------------------
        const int s = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
        const int tile_q = it.pair ? s : 0;
        const int first = it.node0 + tile_q * p.npt;                   // the tile's first node
        const int rows = min(p.npt, it.n - first) * p.G;
        const bool live = row < rows, busy = quad * 32 < rows;
        const int node = first + row / p.G, head = it.h * p.G + row % p.G;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t t_scores = tmem + s * kTile + lanes, t_sums = tmem + S::kO + s * D + lanes;
        const int count = T_ > 0 ? (it.pair ? T_ : (T_ - s + 1) >> 1) : 0;
        constexpr float kLift = Lag<T>::kLift;
        const float c = kCap ? kLog2e : p.scale * kLog2e;
        const float lag = Lag<T>::kLag / c;

        if (p.parent && it.begin < it.tree_tiles) {
            for (int j = tid; j < min(it.last, kParents); j += 256) {
                const int up = p.parent[it.i0 + j];
                parents[j] = (int16_t)(up < -1 || up >= j ? -1 : up);
            }
            named_sync(1, 256);
        }
        int walk = live ? node : -1;
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int k = 0; k < count; ++k) {
            const int tile = it.pair ? k : 2 * k + s, t = it.begin + tile;
            const bool tree = t < it.tree_tiles;
            const int valid = tile_valid(p, it, t);
            if (tree || (valid & 15)) {
                const int pos = 2 * tile + 1;
                ok = ok && mbar_wait_bounded(slot_full(pos % S::kSlots), (pos / S::kSlots) & 1);
                if (!ok) break;
                clean_values<T>(slot_at(pos), row, valid, tree, D / 8, seen);
                fence_proxy_async();
            }
            ok = mbar_wait_bounded(scores_full(s), k & 1);
            if (!ok) break;
            tc_fence_after();
            if (busy) {
                float x[kTile];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j * 32 < valid) tmem_ld32(t_scores + j * 32, x + j * 32);
                    else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[j * 32 + i] = 0.f;        // masked below
                    }
                }
                tmem_wait_ld();
                if (kCap) cap_scores<kTile>(x, p.scale, p.cap);
                if (tree || valid < kTile) {
                    uint32_t see[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int left = valid - j * 32;
                        see[j] = tree ? 0u : left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1 : 0u;
                    }
                    if (tree) {
                        const int t0 = tree_tile_start(it, t);
                        if (!p.parent) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int left = node + 1 - t0 - j * 32;
                                see[j] = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1 : 0u;
                            }
                        } else while (walk >= t0) {
                            const int at = walk - t0;
                            if (at < kTile) {
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (at >> 5 == j) see[j] |= 1u << (at & 31);
                            }
                            walk = up_from(p, it, parents, walk);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kTile; ++i) x[i] = see[i >> 5] >> (i & 31) & 1 ? x[i] : -INFINITY;
                }
                float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                for (int i = 4; i < kTile; i += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        top[k] = i + 4 + k < kTile ? fmaxf(fmaxf(top[k], x[i + k]), x[i + 4 + k]) : fmaxf(top[k], x[i + k]);
                const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(fmaxf(top[2], top[3]), -INFINITY));
                const bool grow = mx > m + lag || (m == -INFINITY && mx > m);
                if (__any_sync(0xffffffffu, grow)) {
                    const float old = m;
                    m = fmaxf(m, mx);
                    const float f = old == -INFINITY ? 0.f : ex2((old - m) * c);
                    l *= f;
                    if (k > 0) {
#pragma unroll
                        for (int j = 0; j < D / 32; ++j) {
                            float o[32];
                            tmem_ld32(t_sums + j * 32, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] *= f;
                            tmem_st32(t_sums + j * 32, o);
                        }
                    }
                }
                const float shift = (m == -INFINITY ? 0.f : m * c) - kLift;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j * 32 < valid) {
                        uint32_t packed[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float2 e = ffma2(make_float2(x[j * 32 + 2 * i], x[j * 32 + 2 * i + 1]), make_float2(c, c), make_float2(-shift, -shift));
                            e.x = ex2(e.x);
                            e.y = ex2(e.y);
                            sum[i & 1] = fadd2(sum[i & 1], e);
                            packed[i] = pack2<T>(e.x, e.y);
                        }
                        tmem_st16(t_scores + j * 16, packed);
                    }
                }
                sum[0] = fadd2(sum[0], sum[1]);
                l += sum[0].x + sum[0].y;
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(probs_ready(s));
        }
        // ---- what came of it ------------------------------------------------------------------------
        ml[s * kTile + row] = make_float2(m, l);
        const int other_count = T_ > 0 ? (T_ - (s ^ 1) + 1) >> 1 : 0;
        if (count > 0) ok = ok && mbar_wait_bounded(sums_full(s), 0);
        if (!it.pair && other_count > 0) ok = ok && mbar_wait_bounded(sums_full(s ^ 1), 0);
        if (!ok) *failed = 1;
        named_sync(1, 256);
        tc_fence_after();
        const bool sick = *seen != 0;
        // a pair of tiles: this stream's; else the two streams' sums of one tile, half the columns each
        float w0 = 0.f, w1 = 0.f;              // what the own (pair) or stream 0's and stream 1's sums count
        if (it.pair) {
            w0 = count > 0 ? 1.f : 0.f;
        } else {
            const float2 a = ml[row], b = ml[kTile + row];
            const bool has_b = T_ > 1;
            m = has_b ? fmaxf(a.x, b.x) : a.x;
            w0 = T_ > 0 && a.x > -INFINITY ? ex2((a.x - m) * c) : 0.f;
            w1 = has_b && b.x > -INFINITY ? ex2((b.x - m) * c) : 0.f;
            l = w0 * a.y + (has_b ? w1 * b.y : 0.f);
            if (T_ == 0) l = 0.f;
        }
        const int64_t out_at = (it.i0 + node) * p.out_row + head * p.out_head;
        const float inv = p.split > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
        const uint32_t own = tmem + S::kO + lanes;
        constexpr int kChunks = D / 32;
        const int j0 = it.pair ? 0 : s * (kChunks / 2), j1 = it.pair ? kChunks : j0 + kChunks / 2;
        if (busy) {
            for (int j = j0; j < j1; ++j) {
                float o[32];
                const bool any0 = it.pair ? count > 0 : T_ > 0, any1 = !it.pair && T_ > 1;
                if (any0) {
                    tmem_ld32(own + (it.pair ? s * D : 0) + j * 32, o);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = any0 ? o[i] * w0 * inv : 0.f;
                if (any1) {
                    float o1[32];
                    tmem_ld32(own + D + j * 32, o1);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = fmaf(o1[i], w1 * inv, o[i]);
                }
                if (sick && live) {
                    // values that are not finite, to the nodes that see them
                    for (int a = node; a >= 0; a = up_from(p, it, parents, a)) {
                        const T *v = reinterpret_cast<const T *>(p.tree_v_at) + (it.i0 + a) * p.tree_row + it.h * p.tree_head + j * 32;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float y = (float)v[i];
                            if (!(fabsf(y) < INFINITY)) o[i] += y;
                        }
                    }
                }
                if (live) {
                    if (p.split == 1) {
                        T *const to = reinterpret_cast<T *>(p.out) + out_at + j * 32;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            reinterpret_cast<uint4 *>(to)[i] =
                                make_uint4(pack2<T>(o[8 * i], o[8 * i + 1]), pack2<T>(o[8 * i + 2], o[8 * i + 3]),
                                           pack2<T>(o[8 * i + 4], o[8 * i + 5]), pack2<T>(o[8 * i + 6], o[8 * i + 7]));
                    } else {
                        float4 *const to = reinterpret_cast<float4 *>(base + S::kRing) + (tile_q * kTile + row) * (D / 4);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            to[(j * 8 + i) ^ (row & 15)] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                }
            }
        }
        const float ln_lift = kLift * kLn2;
        if (it.pair || s == 0) {
            if (p.split == 1) {
                if (live && p.lse)
                    p.lse[(it.i0 + node) * p.Hq + head] = l == 0.f ? -INFINITY : (m * c) * kLn2 + (logf(l) - ln_lift);
            }
        }
        if (p.split > 1) {
            named_sync(1, 256);                         // everyone has read ml
            if (it.pair || s == 0) ml[tile_q * kTile + row] = make_float2(m, l);
        }
    }
    if (p.split > 1) {
        // ---- the cluster's partial results ------------------------------------------------------------
        cluster_arrive();
        cluster_wait();
        if (it.work) {
            constexpr float kLift = Lag<T>::kLift;
            const float c = kCap ? kLog2e : p.scale * kLog2e;
            const int tiles = it.pair ? 2 : 1;
            const int nodes = min(it.n - it.node0, tiles * p.npt), all = nodes * p.G;
            for (int e = rank * 256 + tid; e < all * (D / 4); e += p.split * 256) {
                const int r = e / (D / 4), u = e - r * (D / 4);
                const int tile_q = r / (p.npt * p.G), row = r - tile_q * p.npt * p.G;
                const uint32_t ml_at = smem + S::kMl + (tile_q * kTile + row) * 8;
                const uint32_t o_at = smem + S::kRing + ((tile_q * kTile + row) * (D / 4) + (u ^ (row & 15))) * 16;
                float2 part[kMaxSplit];
                float m = -INFINITY;
#pragma unroll
                for (int k = 0; k < kMaxSplit; ++k)
                    if (k < p.split) {
                        part[k] = cluster_ld2(cluster_address(ml_at, k));
                        m = fmaxf(m, part[k].x);
                    }
                float l = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < kMaxSplit; ++k)
                    if (k < p.split && part[k].x > -INFINITY) {
                        const float w = ex2((part[k].x - m) * c);
                        const float4 v = cluster_ld4(cluster_address(o_at, k));
                        l = fmaf(w, part[k].y, l);
                        o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y);
                        o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
                    } else if (k < p.split && part[k].y != part[k].y) {
                        l = part[k].y;                   // NaN scores only
                        o.x = o.y = o.z = o.w = l;
                    }
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const int64_t node = it.i0 + it.node0 + r / p.G;
                const int head = it.h * p.G + r % p.G;
                T *const to = reinterpret_cast<T *>(p.out) + node * p.out_row + head * p.out_head + u * 4;
                *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
                if (u == 0 && p.lse) p.lse[node * p.Hq + head] = l == 0.f ? -INFINITY : (m * c) * kLn2 + (logf(l) - kLift * kLn2);
            }
        }
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before();
    named_sync(0, kWarps * 32);
}

template <typename T, int D, bool kCap>
int launch(const AttnParams &p, int64_t grid, cudaStream_t stream) {
    auto kernel = tree_attention<T, D, kCap>;
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), Shape<D>::kDynamic);
    if (e == cudaSuccess)
        e = launch_clusters(kernel, (unsigned)p.split, (unsigned)grid, kWarps * 32u, Shape<D>::kDynamic, stream, p);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { record_cuda_error(e); return SSD_ERR_CUDA; }
    return SSD_OK;
}

}  // namespace

bool encode_map(CUtensorMap *map, ssd_dtype dtype, const void *base, int rank, const uint64_t *dims,
                const uint64_t *strides, const uint32_t *box) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    if (!encode) { cudaGetLastError(); record_cuda_error(cudaErrorNotSupported); return false; }
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(map, dtype == SSD_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                              (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { record_cuda_error(cudaErrorInvalidValue); return false; }
    return true;
}

bool encode_rows(CUtensorMap *map, ssd_dtype dtype, const ssd_heads &x, int D, int64_t M, int box_heads, int box_rows) {
    // an axis of one entry may come with any stride: the map gets one that it can hold
    const uint64_t dims[3] = {(uint64_t)D, (uint64_t)x.heads, (uint64_t)M};
    const uint64_t strides[2] = {2ull * (x.heads > 1 ? x.head_stride : D), 2ull * (M > 1 ? x.row_stride : (int64_t)x.heads * D)};
    const uint32_t box[3] = {64, (uint32_t)box_heads, (uint32_t)box_rows};
    return encode_map(map, dtype, x.data, 3, dims, strides, box);
}
bool encode_cache(CUtensorMap *map, const ssd_kv_cache &c, const void *data, int box) {
    const uint64_t dims[4] = {(uint64_t)c.head_dim, (uint64_t)c.heads, (uint64_t)c.page_size, (uint64_t)(c.pages > 0 ? c.pages : 1)};
    const uint64_t strides[3] = {2ull * (c.heads > 1 ? c.head_stride : c.head_dim), 2ull * (c.page_size > 1 ? c.slot_stride : c.head_dim),
                                 2ull * (c.pages > 1 ? c.page_stride : c.head_dim)};
    const uint32_t b[4] = {64, 1, (uint32_t)box, 1};
    return encode_map(map, c.dtype, data, 4, dims, strides, b);
}

int launch_tree_attention(const ssd_heads &q, const ssd_heads &tree_k, const ssd_heads &tree_v, const ssd_kv_cache &cache,
                          const int64_t *tok_off, const int32_t *parent, int B, int64_t M, int max_nodes, float scale,
                          float cap, const ssd_heads &out, float *lse, uint32_t *status, cudaStream_t stream) {
    if (B == 0) return SSD_OK;
    AttnParams p;
    p.paging = paging(cache.page_size);
    p.G = q.heads / cache.heads;
    p.npt = kTile / p.G;
    if (p.npt > max_nodes) p.npt = max_nodes > 0 ? max_nodes : 1;      // no more of q is fetched than a tree can have
    const int D = cache.head_dim;
    if (M > 0) {
        if (!encode_rows(&p.q, cache.dtype, q, D, M, p.G, p.npt) || !encode_rows(&p.tree_k, cache.dtype, tree_k, D, M, 1, kTreeBox) ||
            !encode_rows(&p.tree_v, cache.dtype, tree_v, D, M, 1, kTreeBox))
            return SSD_ERR_CUDA;
    }
    if (cache.pages > 0 && (!encode_cache(&p.cache_k, cache, cache.k, p.paging.box) || !encode_cache(&p.cache_v, cache, cache.v, p.paging.box)))
        return SSD_ERR_CUDA;
    p.table = cache.page_table; p.len = cache.len; p.parent = parent; p.off = tok_off;
    p.tree_v_at = tree_v.data; p.tree_row = tree_v.row_stride; p.tree_head = tree_v.head_stride;
    p.out = out.data; p.out_row = out.row_stride; p.out_head = out.head_stride;
    p.lse = lse; p.status = status; p.table_stride = cache.table_stride; p.M = M;
    p.B = B; p.Hq = q.heads; p.Hkv = cache.heads;
    p.q_items = max_nodes > p.npt ? (max_nodes + 2 * p.npt - 1) / (2 * p.npt) : 1;
    p.max_nodes = max_nodes; p.n_pages = cache.pages;
    p.max_pages = cache.pages > 0 ? cache.max_pages : 0;      // without pages every cache is empty
    p.scale = scale; p.cap = cap;
    const int sms = device_sm_count();
    if (sms <= 0) return SSD_ERR_CUDA;
    const int64_t items = (int64_t)B * p.Hkv * p.q_items;
    const int64_t tiles = 1 + ((int64_t)p.max_pages * cache.page_size + kTile - 1) / kTile;
    p.split = 1;
    while (p.split < kMaxSplit && items * p.split * 2 <= sms && p.split * 2 <= tiles) p.split *= 2;
    const int64_t grid = items * p.split;
    if (grid > INT32_MAX) return SSD_ERR_ARG;
    const bool half = cache.dtype == SSD_F16;
    if (D == 64)
        return half ? (cap > 0.f ? launch<__half, 64, true>(p, grid, stream) : launch<__half, 64, false>(p, grid, stream))
                    : (cap > 0.f ? launch<__nv_bfloat16, 64, true>(p, grid, stream) : launch<__nv_bfloat16, 64, false>(p, grid, stream));
    return half ? (cap > 0.f ? launch<__half, 128, true>(p, grid, stream) : launch<__half, 128, false>(p, grid, stream))
                : (cap > 0.f ? launch<__nv_bfloat16, 128, true>(p, grid, stream) : launch<__nv_bfloat16, 128, false>(p, grid, stream));
}

}  // namespace ssd
