// Attention for draft trees over a paged key/value cache (ssd_tree_attention).
//
// Every node of an utterance's tree attends to the utterance's cache and to its own line of
// descent: out_i = sum_j softmax_j(s_ij) v_j with s_ij = scale q_i.k_j, or cap tanh(scale q_i.k_j / cap).
// The query heads that share a kv head are rows of one product: a tile is 128 / G nodes by G heads, its
// keys come 128 at a time, and the softmax is carried as a running maximum and sum per row.
//
// An item is one kv head of one utterance and up to two tiles of its queries; one pass over the item's keys
// serves both tiles, or, where the rows fill one tile or less, its key tiles alternate between two
// accumulators.  Either way there are two streams of (scores -> softmax -> product), so the tensor
// cores work on one while the other's exponentials are taken: warps 0-3 and 4-7 hold one row a thread, warps
// 8 and 10 issue the copies, warp 9 the products, and warp 11 keeps the work coming.
// Scores and accumulators live in tensor memory; probabilities go back there in 16 bits, over the
// scores they came from, and are the first operand of the second product.
//
// All items' key tiles form one line, which is cut into as many equal parts as there are multiprocessors: one
// CTA each, whose pipeline runs on from item to item.  Lengths may be as ragged as they like, and few
// items over long caches fill the device as well as many over short ones.  An item that a cut goes through
// leaves partial results (unscaled sums, maxima and sums of probabilities, fp32) in the workspace, which a
// closing kernel joins.
//
// Measured (32 query and 8 kv heads of 128, bf16, pages of 16): trees of 5 to 32 nodes on 64 caches of 500 to
// 3,000 slots 119 us, 475 MB at 4.0 TB/s; chains of 50 to 200 nodes on 128 caches of 250 to 1,500 slots 488 us, 256 GFLOP at
// 523 TFLOP/s.  (Comments below give times before and after a step on one box each; boxes differ by up to 15 % where the
// power limit is reached.)  A key tile takes a CTA 2,400 clocks either way: at few rows that is what HBM gives a
// multiprocessor, at many it is the cycle scores -> softmax -> product of a stream (4,500 clocks) over two streams, of
// which the products are 1,220 and the softmax 2,250.
#include <math.h>

#include <atomic>

#include "ssd_ranges.cuh"
#include "ssd_tc.cuh"

namespace ssd {
namespace {

using namespace tc;

constexpr int kWarps = 12, kLaunchRegisters = 168;
constexpr int kParents = 256;            // parents kept in shared memory; more are read from global
constexpr int kTreeBox = 16;             // nodes that one copy brings

// What a CTA leaves for the closing kernel: the part of an item that begins before it (`head`) and
// that of one which goes on behind it (`tail`).
struct Cut {
    int32_t head;                        // 0: none; 1: goes on; 2: ends here
    int32_t tail;                        // 1: there is one
    int32_t b, h, node0, rows;           // the tail's item
    int32_t failed;                      // whether a wait of its ran out
};

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
    Cut *cuts;                           // [grid]
    float *parts;                        // [grid][2] x (rows pairs of maximum and sum, rows x D sums)
    int part_rows;
    int B, Hq, Hkv, G, npt, max_nodes, n_pages, max_pages;
    Paging paging;
    float scale, cap;
};
__host__ __device__ inline int64_t part_floats(int rows, int D) { return (int64_t)rows * (D + 2); }

template <int D> struct Shape {
    static constexpr int kBlocks = D / 64;
    static constexpr int kSlotBytes = kBlocks * kBlockBytes;      // a tile of keys or of values
    static constexpr int kSlots = D == 128 ? 5 : 8;
    static constexpr int kRing = 2 * kSlotBytes;                  // behind the two tiles of queries
    static constexpr int kMisc = kRing + kSlots * kSlotBytes;
    static constexpr int kBars = kMisc;     // full[], empty[], q full[2], q empty[2], scores[2], probs[2], sums[2], sums free[2]
    static constexpr int kNumBars = 2 * kSlots + 17;              // and segments full[2], empty[2], softmax warps together
    static constexpr int kWords = kBars + kNumBars * 8;           // tmem address, failed, bad value seen [2]
    static constexpr int kMl = (kWords + 16 + 15) / 16 * 16;      // [2][128] running maximum and sum
    static constexpr int kParent = kMl + 2 * kTile * 8;
    static constexpr int kSegments = (kParent + kParents * 2 + 15) / 16 * 16;
    static constexpr int kGroups = kSegments + 2 * 64;            // groups of 16 keys in a slot
    static constexpr int kBytes = kGroups + kSlots * 4;
    static constexpr int kO = 256;                                // tensor memory: scores at 0 and 128, sums here
};
static_assert(Shape<128>::kBytes <= 232448, "shared memory");

// ---- the line of key tiles and its cuts -----------------------------------------------------------
// A tile costs as much as it has tiles of queries, 2,400 clocks each; an item's end costs 6,000 to 8,000 (its last products
// are waited for, its results written).
constexpr int kEndCost = 3, kLeastPart = 2;
struct Utterance {
    int64_t i0;
    int n, len, cache_tiles, q_items;
};
__device__ __forceinline__ Utterance utterance(const AttnParams &p, int b) {
    Utterance u;
    u.i0 = p.off[b];
    const int64_t i1 = p.off[b + 1];
    const int len = p.len[b];
    const bool ok = !(u.i0 < 0 || i1 < u.i0 || i1 > p.M || i1 - u.i0 > p.max_nodes);
    u.n = ok ? (int)(i1 - u.i0) : 0;
    const int64_t room = (int64_t)p.max_pages * p.paging.page;
    u.len = min(max(len, 0), (int)min(room, kMostSlots));
    u.cache_tiles = paged_tiles(p.paging, u.len);
    u.q_items = (u.n + 2 * p.npt - 1) / (2 * p.npt);
    return u;
}
struct Item {
    int node0;           // its first node
    int pair;            // 1: two tiles of queries
    int last;            // one past the last node that is a key
    int tree_tiles, tiles;
};
__device__ __forceinline__ Item item_of(const AttnParams &p, const Utterance &u, int qi) {
    Item it;
    it.node0 = qi * 2 * p.npt;
    it.pair = u.n - it.node0 > p.npt;
    it.last = min(u.n, it.node0 + 2 * p.npt);
    it.tree_tiles = (it.last + kTile - 1) / kTile;
    it.tiles = it.tree_tiles + u.cache_tiles;
    return it;
}
__device__ __forceinline__ int64_t cost(const Item &it) { return (int64_t)it.tiles * (1 + it.pair) + kEndCost; }
__device__ __forceinline__ int64_t cost(const AttnParams &p, const Utterance &u) {     // of one head
    int64_t c = 0;
    for (int qi = 0; qi < u.q_items; ++qi) c += cost(item_of(p, u, qi));
    return c;
}

// What a CTA works on next: tiles [begin, end) of an item.  One warp walks the line and keeps two of
// these ahead of the others in shared memory.
struct Segment {
    int64_t i0;
    int b, h, n, len;
    int node0, pair, last, tree_tiles, tiles;
    int begin, end;      // begin == end: no more
    int pad[3];
};
static_assert(sizeof(Segment) == 64, "");

// The CTA's part of the line [lo, hi), where in it the walk stands, and its next segment.
struct Walk {
    Utterance u;
    Item it;
    int64_t lo, hi, at;  // at: where the current item begins
    int b, h, qi, begin, end;
    __device__ __forceinline__ bool cut_item(const AttnParams &p) {
        it = item_of(p, u, qi);
        const int64_t from = lo - at, to = hi - at;      // tile k lies at at + k (1 + pair)
        begin = from <= 0 ? 0 : (int)min((from + it.pair) >> it.pair, (int64_t)it.tiles);
        end = to <= 0 ? 0 : (int)min((to + it.pair) >> it.pair, (int64_t)it.tiles);
        return begin < end;
    }
    __device__ __forceinline__ bool next(const AttnParams &p) {
        do {
            at += cost(it);
            if (at >= hi) return false;
            if (++qi == u.q_items) {
                qi = 0;
                if (++h == p.Hkv) {
                    h = 0;
                    do {
                        if (++b >= p.B) return false;
                        u = utterance(p, b);
                    } while (u.n == 0);
                }
            }
        } while (!cut_item(p));
        return true;
    }
    // a b / c, in 32 bits where they are enough (they nearly always are, and a division of 64 is a hundred instructions)
    static __device__ __forceinline__ int64_t scaled(int64_t a, int b, int c) {
        return a < (1 << 20) ? (int64_t)((uint32_t)a * (uint32_t)b / (uint32_t)c) : a * b / c;      // b is below 2^12: a grid
    }
    // By one warp: costs[b] are the utterances' (of one head), the first `held` of them.
    __device__ __forceinline__ bool first(const AttnParams &p, const int64_t *costs, int held, int lane) {
        auto head_cost = [&](int i) { return i >= p.B ? 0 : i < held ? costs[i] : cost(p, utterance(p, i)); };
        const int64_t mine = head_cost(lane);
        int64_t total = mine;
        for (int i = lane + 32; i < p.B; i += 32) total += head_cost(i);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        total *= p.Hkv;
        // parts of at least kLeastPart: what a short one saves, the closing kernel spends on joining it
        const int parts = (int)min((int64_t)gridDim.x, max(total / kLeastPart, (int64_t)1));
        if ((int)blockIdx.x >= parts) return false;
        lo = scaled(total, blockIdx.x, parts);
        hi = scaled(total, blockIdx.x + 1, parts);
        if (lo >= hi) return false;
        int64_t before = 0;
        for (int i0 = 0; i0 < p.B; i0 += 32) {
            const int64_t one = i0 ? head_cost(i0 + lane) : mine, v = one * p.Hkv;
            int64_t x = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            const unsigned here = __ballot_sync(0xffffffffu, lo < before + x);
            if (here) {
                const int who = __ffs(here) - 1;         // lo lies in utterance i0 + who
                b = i0 + who;
                u = utterance(p, b);
                const int64_t each = __shfl_sync(0xffffffffu, one, who);
                at = before + __shfl_sync(0xffffffffu, x - v, who);
                const int64_t in = lo - at;
                h = in < (1ll << 31) && each < (1ll << 31) ? (int)((uint32_t)in / (uint32_t)each) : (int)(in / each);
                at += h * each;
                for (qi = 0; qi + 1 < u.q_items; ++qi) {
                    const int64_t c = cost(item_of(p, u, qi));
                    if (lo < at + c) break;
                    at += c;
                }
                return cut_item(p) || next(p);
            }
            before += __shfl_sync(0xffffffffu, x, 31);
        }
        return false;
    }
};
// The tree's own tiles come first, last nodes first: a thread walks its node's line upwards once.
__device__ __forceinline__ int tree_tile_start(const volatile Segment &g, int t) { return (g.tree_tiles - 1 - t) * kTile; }
__device__ __forceinline__ int tile_valid(const AttnParams &p, const volatile Segment &g, int t) {
    if (t < g.tree_tiles) return min(kTile, g.last - tree_tile_start(g, t));
    return paged_tile(p.paging, g.len, t - g.tree_tiles).valid;
}

// The status of utterance b, by one warp.
__device__ __forceinline__ void report(const AttnParams &p, int b, int lane) {
    const Utterance u = utterance(p, b);
    const int64_t i1 = p.off[b + 1];
    uint32_t bits = 0;
    if (u.i0 < 0 || i1 < u.i0 || i1 > p.M || i1 - u.i0 > p.max_nodes) bits |= SSD_UTT_BAD_OFFSETS;
    if (p.len[b] != u.len) bits |= SSD_UTT_BAD_CACHE;
    if (p.parent)
        for (int j = lane; j < u.n; j += 32) {
            const int up = p.parent[u.i0 + j];
            if (up < -1 || up >= j) bits |= SSD_UTT_BAD_PARENT;
        }
    const int pages = u.n > 0 ? (int)(((int64_t)u.len + p.paging.page - 1) / p.paging.page) : 0;
    for (int j = lane; j < pages; j += 32) {
        const int id = p.table[b * p.table_stride + j];
        if (id < 0 || id >= p.n_pages) bits |= SSD_UTT_BAD_CACHE;
    }
    bits = __reduce_or_sync(0xffffffffu, bits);
    if (lane == 0) p.status[b] = bits;
}

__device__ __forceinline__ int up_from(const AttnParams &p, int64_t i0, const int16_t *parents, int j) {
    if (!p.parent) return j - 1;
    if (parents && j < kParents) return parents[j];
    const int up = p.parent[i0 + j];
    return up < -1 || up >= j ? -1 : up;
}

// The product runs over whole groups of 16 keys, and 0 times NaN is NaN: values behind the last key
// are made zeros, and so are the tree's own values that are not finite (a node that does not see them
// must not get them; `seen` says that there are some, and those that do see them get them at the end).
template <typename T, int D>
__device__ __forceinline__ void clean_values(uint32_t tile, int row, int valid, bool tree, volatile uint32_t *seen) {
    if (row >= valid) {
        if (row < (valid + 15) / 16 * 16)
#pragma unroll
            for (int u = 0; u < D / 8; ++u)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(unit_at(tile, row, u)), "r"(0) : "memory");
        return;
    }
    if (!tree) return;
    constexpr uint32_t e = Format<T>::kExponent * 0x10001u;
    uint32_t bad = 0;                        // a bit for every 4 units that hold something with all exponent bits set
#pragma unroll
    for (int u0 = 0; u0 < D / 8; u0 += 4) {
        uint32_t w[16], hit = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                         : "r"(unit_at(tile, row, u0 + i)));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t t = ~w[i] & e;    // a half of zeros: all exponent bits set
            hit |= (t - 0x00010001u) & ~t & 0x80008000u;
        }
        if (hit) bad |= 1u << (u0 / 4);
    }
    if (bad == 0) return;
    *seen = 1;
    __threadfence_block();
    for (int u = 0; u < D / 8; ++u) {
        if (!(bad >> (u / 4) & 1)) continue;
        uint32_t w[4];
        const uint32_t at = unit_at(tile, row, u);
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t t = ~w[i] & e;
            w[i] &= (t & 0xffffu ? 0xffffu : 0u) | (t >> 16 ? 0xffff0000u : 0u);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
}

// N lanes' rows of N 16-byte units each, turned so that a store of the warp writes N units of a row side by side:
// before, lane i has unit j of row i in v[j]; after, unit i of row j (of its group of N lanes).
template <int N> __device__ __forceinline__ void turn(uint4 *v) {
    const int lane = threadIdx.x & (N - 1);
#pragma unroll
    for (int o = 1; o < N; o <<= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (j & o) continue;
            // lanes without the bit give v[j | o] and take the partner's v[j], and the other way round
            uint4 a = up ? v[j] : v[j | o];
            a.x = __shfl_xor_sync(0xffffffffu, a.x, o);
            a.y = __shfl_xor_sync(0xffffffffu, a.y, o);
            a.z = __shfl_xor_sync(0xffffffffu, a.z, o);
            a.w = __shfl_xor_sync(0xffffffffu, a.w, o);
            if (up) v[j] = a; else v[j | o] = a;
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

    auto slot_full = [&](int slot) { return smem + S::kBars + 8 * slot; };
    auto slot_empty = [&](int slot) { return smem + S::kBars + 8 * (S::kSlots + slot); };
    const uint32_t more = smem + S::kBars + 16 * S::kSlots;
    auto q_full = [&](int i) { return more + 8 * i; };
    auto q_empty = [&](int i) { return more + 16 + 8 * i; };
    auto scores_full = [&](int s) { return more + 32 + 8 * s; };
    auto probs_ready = [&](int s) { return more + 48 + 8 * s; };
    auto sums_full = [&](int s) { return more + 64 + 8 * s; };
    auto sums_free = [&](int s) { return more + 80 + 8 * s; };
    auto segment_full = [&](int i) { return more + 96 + 8 * i; };
    auto segment_empty = [&](int i) { return more + 112 + 8 * i; };
    const uint32_t together = more + 128;
    volatile Segment *const ring = reinterpret_cast<volatile Segment *>(base + S::kSegments);
    volatile uint32_t *const words = reinterpret_cast<volatile uint32_t *>(base + S::kWords);
    volatile uint32_t *const failed = words + 1;
    float2 *const ml = reinterpret_cast<float2 *>(base + S::kMl);
    int16_t *const parents = reinterpret_cast<int16_t *>(base + S::kParent);
    volatile int *const groups_of = reinterpret_cast<volatile int *>(base + S::kGroups);
    auto slot_at = [&](int slot) { return smem + S::kRing + slot * S::kSlotBytes; };

    if (warp == 8) tmem_alloc(smem + S::kWords, 512);
    if (tid == 0) {
        for (int i = 0; i < S::kSlots; ++i) { mbar_init(slot_full(i), 1); mbar_init(slot_empty(i), 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full(s), 1);
            mbar_init(q_empty(s), 1);
            mbar_init(scores_full(s), 1);
            mbar_init(probs_ready(s), 4);
            mbar_init(sums_free(s), 8);
            mbar_init(sums_full(s), 1);
            mbar_init(segment_full(s), 1);
            mbar_init(segment_empty(s), 11);
        }
        mbar_init(together, 8);
        mbar_init_fence();
        words[1] = words[2] = words[3] = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = words[0];
    pdl_wait();
    // what the utterances cost, in front of the walk (in the queries' place, which are not there yet)
    constexpr int kHeld = 2 * S::kSlotBytes / 8;
    int64_t *const costs = reinterpret_cast<int64_t *>(base);
    for (int b = tid; b < min(p.B, kHeld); b += kWarps * 32) costs[b] = cost(p, utterance(p, b));
    fence_proxy_async();
    __syncthreads();
    // The i-th segment, read in place by whole warps: `take` waits for it, `give` hands its place back.
    auto take = [&](int i, bool &ok) {
        ok = ok && mbar_wait_bounded(segment_full(i & 1), i >> 1 & 1);
        return ok && ring[i & 1].begin < ring[i & 1].end;
    };
    auto give = [&](int i) {
        __syncwarp();
        if (lane == 0) mbar_arrive(segment_empty(i & 1));
    };

    if (warp >= 8) {
        // of the 168 registers a thread is launched with, softmax threads get 224 and these keep 56
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        bool ok = true;
        if (warp == 8 || warp == 10) {
            // ---- copies: queries and keys, and values, a warp each (it is the issue of many small copies
            // that takes time, so every lane issues one)
            const int kv = warp == 10, page_count = p.paging.pages ? p.paging.pages : 1;
            // Few rows leave a tile's time to these two warps.  Its place in the ring is counted along, its place in the
            // cache worked out and its pages looked up a turn ahead: eight caches of 20,000 slots 133 -> 129 us, trees
            // 107 -> 106.
            int slot = kv, round = 0;                                // keys and values take turns
            int used[2] = {0, 0}, buffer = 0;
            const int i = lane / S::kBlocks, x = lane % S::kBlocks;  // copies are of 64 columns and 8 rows at least: a lane for each
            for (int g = 0; take(g, ok); give(g++)) {
                const volatile Segment &w = ring[g & 1];
                const int begin = w.begin, end = w.end, tree_tiles = w.tree_tiles, last = w.last, h = w.h, len = w.len, i0 = (int)w.i0;
                if (!kv) {
                    for (int j = 0; j < 1 + w.pair && ok; ++j) {
                        const int q = w.pair ? j : buffer;
                        if (used[q] > 0) ok = mbar_wait_bounded(q_empty(q), (used[q] - 1) & 1);
                        if (!ok) break;
                        ++used[q];
                        if (lane == 0) mbar_arrive_expect_tx(q_full(q), S::kBlocks * p.G * p.npt * 128);
                        __syncwarp();
                        if (lane < S::kBlocks)
                            tma_load_3d(smem + q * S::kSlotBytes + lane * kBlockBytes, &p.q, lane * 64, h * p.G,
                                        i0 + w.node0 + j * p.npt, q_full(q));
                    }
                    if (!w.pair) buffer ^= 1;
                }
                const int32_t *const table = p.table + w.b * p.table_stride;
                auto where = [&](int t) { return t < tree_tiles ? TileAt{0, 0, 0} : paged_tile(p.paging, len, t - tree_tiles); };
                // Lane i: the tile's i-th page, as the table has it.  It is looked at in the next turn of the loop.
                auto page_id = [&](int t, const TileAt &a) {
                    return t < tree_tiles || t >= end || lane >= page_count ? 0 : a.page + lane < p.max_pages ? table[a.page + lane] : -1;
                };
                TileAt next_at = where(begin);
                int next = page_id(begin, next_at);
                for (int t = begin; t < end; ++t) {
                    const TileAt tile = next_at;
                    const int id = next < 0 || next >= p.n_pages ? p.n_pages : next;     // outside: the copy fills in zeros
                    next_at = where(t + 1);
                    next = page_id(t + 1, next_at);
                    const bool tree = t < tree_tiles;
                    const int t0 = (tree_tiles - 1 - t) * kTile, valid = tree ? min(kTile, last - t0) : tile.valid;
                    const int box = tree ? kTreeBox : p.paging.box, copies = (valid + box - 1) / box;
                    ok = mbar_wait_bounded(slot_empty(slot), ~round & 1);             // a new barrier lets the first round pass
                    if (!ok) break;
                    const uint32_t bar = slot_full(slot);
                    if (lane == 0) {
                        groups_of[slot] = (valid + 15) >> 4;
                        mbar_arrive_expect_tx(bar, copies * box * 128 * S::kBlocks);
                    }
                    const int page = __shfl_sync(0xffffffffu, id, p.paging.pages ? i : 0);
                    if (i < copies) {
                        const uint32_t dst = slot_at(slot) + x * kBlockBytes + i * box * 128;
                        if (tree)
                            tma_load_3d(dst, kv ? &p.tree_v : &p.tree_k, x * 64, h, i0 + t0 + i * box, bar);
                        else
                            tma_load_4d(dst, kv ? &p.cache_v : &p.cache_k, x * 64, h, p.paging.pages ? 0 : tile.slot + i * box, page, bar);
                    }
                    slot += 2;
                    if (slot >= S::kSlots) slot -= S::kSlots, ++round;
                }
            }
        } else if (warp == 9) {
            // ---- products -----------------------------------------------------------------------
            const uint32_t tm = uniform(tmem);
            int pos0 = 0, used[2] = {0, 0}, buffer = 0, done[2] = {0, 0};
            for (int g = 0; take(g, ok); give(g++)) {
                const volatile Segment &w = ring[g & 1];
                const int pair = uniform(w.pair), tiles = uniform(w.end - w.begin);
                const int units = pair ? 2 * tiles : tiles;
                for (int i = 0; i < 1 + pair && ok; ++i) {
                    const int q = pair ? i : buffer;
                    ok = mbar_wait_bounded(q_full(q), used[q]++ & 1);
                }
                // (stream, tile) pairs in the order of their products: u is of stream u & 1
                auto scores = [&](int u) {                                                // the groups of 16 keys it covers
                    const int s = u & 1, tile = pair ? u >> 1 : u, pos = pos0 + 2 * tile, q = pair ? s : buffer;
                    ok = ok && mbar_wait_bounded(slot_full(pos % S::kSlots), (pos / S::kSlots) & 1);
                    if (!ok) return 0;
                    const int n16 = uniform(groups_of[pos % S::kSlots]);
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t idesc = instruction<T>(n16 * 16, false);
                        const uint64_t a = operand(smem + q * S::kSlotBytes), k = operand(slot_at(pos % S::kSlots));
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const int at = (x >> 2) * (kBlockBytes >> 4) + (x & 3) * 2;   // 16 columns = 32 bytes of a block's rows
                            mma_ss(tm + s * kTile, a + at, k + at, idesc, x > 0);
                        }
                        mma_commit(scores_full(s));
                        if (!pair || s) mma_commit(slot_empty(pos % S::kSlots));
                        if (tile == tiles - 1) mma_commit(q_empty(q));
                    }
                    __syncwarp();
                    return n16;
                };
                auto values = [&](int u, int n16) {
                    const int s = u & 1, k = u >> 1, tile = pair ? k : u, pos = pos0 + 2 * tile + 1;
                    ok = ok && mbar_wait_bounded(slot_full(pos % S::kSlots), (pos / S::kSlots) & 1);
                    if (k == 0 && g > 0) ok = ok && mbar_wait_bounded(sums_free(s), (g - 1) & 1);
                    ok = ok && mbar_wait_bounded(probs_ready(s), (done[s] + k) & 1);
                    if (!ok) return;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t idesc = instruction<T>(D, true);
                        const uint64_t v = operand(slot_at(pos % S::kSlots));
#pragma unroll
                        for (int x = 0; x < kTile / 16; ++x)                              // 16 keys = 2,048 bytes of a block
                            if (x < n16)
                                mma_ts(tm + S::kO + s * D, tm + s * kTile + x * 8, v + x * (2048 >> 4), idesc, k > 0 || x > 0);
                        if (!pair || s) mma_commit(slot_empty(pos % S::kSlots));
                        if (u + 2 >= units) mma_commit(sums_full(s));
                    }
                    __syncwarp();
                };
                int n0 = ok ? scores(0) : 0, n1 = units > 1 ? scores(1) : 0;
                for (int u = 0; u < units && ok; ++u) {
                    values(u, n0);
                    n0 = n1;
                    if (u + 2 < units) n1 = scores(u + 2);
                }
                done[0] += (units + 1) >> 1;
                done[1] += units >> 1;
                pos0 += 2 * tiles;
                if (!pair) buffer ^= 1;
            }
        } else {
            // ---- the walk along the line ----------------------------------------------------------
            Walk k;
            bool more_work = k.first(p, costs, kHeld, lane);
            // the costs are read: the queries may come (their warp waits for the first segment)
            fence_proxy_async();
            for (int g = 0; ok; ++g) {
                if (g >= 2) ok = mbar_wait_bounded(segment_empty(g & 1), ((g >> 1) - 1) & 1);
                if (!ok) break;
                if (lane == 0) {
                    volatile Segment &n = ring[g & 1];
                    words[2 + (g & 1)] = 0;                       // nobody reads the earlier item's any more
                    n.i0 = k.u.i0;
                    n.b = k.b; n.h = k.h; n.n = k.u.n; n.len = k.u.len;
                    n.node0 = k.it.node0; n.pair = k.it.pair; n.last = k.it.last; n.tree_tiles = k.it.tree_tiles; n.tiles = k.it.tiles;
                    n.begin = more_work ? k.begin : 0;
                    n.end = more_work ? k.end : 0;

                    mbar_arrive(segment_full(g & 1));
                }
                __syncwarp();
                if (!more_work) break;
                more_work = k.next(p);
            }
            for (int b = blockIdx.x; b < p.B; b += gridDim.x) report(p, b, lane);
        }
        if (!ok) *failed = 1;
        named_sync(0, kWarps * 32);
        if (*failed) drain_after_error();
        if (warp == 8) {
            tc_fence_after();
            tmem_free(tmem, 512);
        }
        return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    // ---- softmax ------------------------------------------------------------------------------------
    const int s = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const uint32_t t_scores = tmem + s * kTile + lanes;
    constexpr float kLift = Lag<T>::kLift;
    const float c = kCap ? kLog2e : p.scale * kLog2e;
    const float lag = Lag<T>::kLag / c;
    const int tile_rows = p.npt * p.G;
    bool ok = true;
    int pos0 = 0, done = 0, closed[2] = {0, 0};
    if (tid == 0) p.cuts[blockIdx.x] = Cut{};
    // The eight softmax warps wait for one another, with a limit as every wait here: a warp that has given up
    // keeps nobody.
    int meetings = 0;
    auto meet = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(together);
        ok = ok && mbar_wait_bounded(together, meetings++ & 1);
    };
    for (int g = 0; take(g, ok); give(g++)) {
        const volatile Segment &w = ring[g & 1];
        const int pair = w.pair, begin = w.begin, tiles = w.end - begin;
        const int tile_q = pair ? s : 0;
        const int first = w.node0 + tile_q * p.npt;                 // the tile's first node
        const int rows = min(p.npt, w.n - first) * p.G;
        const bool live = row < rows, busy = quad * 32 < rows;
        const int node = first + row / p.G, head = w.h * p.G + row % p.G;
        const uint32_t t_sums = tmem + S::kO + s * D + lanes;
        const int count = pair ? tiles : (tiles - s + 1) >> 1;
        volatile uint32_t *const seen = words + 2 + (g & 1);

        // A tree of up to 32 nodes: a lane has a node, and five rounds of doubling over the lanes give its line.  Larger
        // ones are walked, from parents in shared memory (5,000 clocks an item where this takes 400).
        const bool small = p.parent && w.last <= 32;
        uint32_t line = 0;
        if (small && begin < w.tree_tiles) {
            int up = lane < w.last ? p.parent[w.i0 + lane] : -1;
            if (up < -1 || up >= lane) up = -1;
            uint32_t mask = 1u << lane;
#pragma unroll
            for (int round = 0; round < 5; ++round) {
                const int from = up < 0 ? lane : up;
                const uint32_t above = __shfl_sync(0xffffffffu, mask, from);
                const int further = __shfl_sync(0xffffffffu, up, from);
                if (up >= 0) { mask |= above; up = further; }
            }
            line = __shfl_sync(0xffffffffu, mask, node & 31);
        }
        if (p.parent && !small && begin < w.tree_tiles) {
            meet();                                  // the earlier item's are read
            for (int j = tid; j < min(w.last, kParents); j += 256) {
                const int up = p.parent[w.i0 + j];
                parents[j] = (int16_t)(up < -1 || up >= j ? -1 : up);
            }
            meet();
        }
        int walk = live ? node : -1;
        float m = -INFINITY, l = 0.f;
        for (int k = 0; k < count; ++k) {
            const int tile = pair ? k : 2 * k + s, t = begin + tile;
            const bool tree = t < w.tree_tiles;
            const int valid = tile_valid(p, w, t);
            ok = mbar_wait_bounded(scores_full(s), (done + k) & 1);
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
                if (kCap) cap_scores<kTile>(x, p.scale, p.cap, live);
                if (tree || valid < kTile) {
                    uint32_t see[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int left = valid - j * 32;
                        see[j] = tree ? 0u : left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1 : 0u;
                    }
                    if (tree) {
                        const int t0 = tree_tile_start(w, t);
                        if (small) {
                            see[0] = line;
                        } else if (!p.parent) {
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
                            walk = up_from(p, w.i0, parents, walk);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (__all_sync(0xffffffffu, see[j] == 0xffffffffu)) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[j * 32 + i] = see[j] >> i & 1 ? x[j * 32 + i] : -INFINITY;
                    }
                }
                float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                for (int i = 4; i < kTile; i += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        top[k] = i + 4 + k < kTile ? fmaxf(fmaxf(top[k], x[i + k]), x[i + 4 + k]) : fmaxf(top[k], x[i + k]);
                const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(fmaxf(top[2], top[3]), -INFINITY));
                const bool grow = live && (mx > m + lag || (m == -INFINITY && mx > m));
                if (__any_sync(0xffffffffu, grow)) {
                    const float old = m;
                    m = fmaxf(m, mx);
                    const float f = old == -INFINITY ? 0.f : ex2((old - m) * c);
                    l *= f;
                    if (k > 0) {
#pragma unroll 1
                        for (int j = 0; j < D / 16; ++j) {       // a few at a time: the scores fill the registers
                            float o[16];
                            tmem_ld16(t_sums + j * 16, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] *= f;
                            tmem_st16(t_sums + j * 16, reinterpret_cast<const uint32_t *>(o));
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
            if (tree || (valid & 15)) {              // by now the values are there
                const int pos = pos0 + 2 * tile + 1, slot = pos % S::kSlots;
                ok = mbar_wait_bounded(slot_full(slot), (pos / S::kSlots) & 1);
                if (!ok) break;
                clean_values<T, D>(slot_at(slot), row, valid, tree, seen);
                fence_proxy_async();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(probs_ready(s));
        }
        done += count;
        pos0 += 2 * tiles;
        // ---- what came of it ------------------------------------------------------------------------
        // A pair's streams have nothing to do with one another: each ends when it does (chains 484 -> 461 us against a
        // meeting, 494 -> 480 on another box).  Those of one tile meet.
        if (!pair) ml[s * kTile + row] = make_float2(m, l);
        const bool any[2] = {true, pair || tiles > 1};                 // whether a stream had tiles
        for (int i = 0; i < 2; ++i)
            if (any[i]) {
                if (!pair || i == s) ok = ok && mbar_wait_bounded(sums_full(i), closed[i] & 1);
                ++closed[i];
            }
        if (!ok) *failed = 1;
        if (!pair) meet();
        tc_fence_after();
        const bool sick = *seen != 0;
        // a pair of tiles: this stream's sums; else the two streams' of one tile, half the columns each
        float w0 = 1.f, w1 = 0.f;
        if (!pair) {
            const float2 a = ml[row], b = ml[kTile + row];
            m = any[1] ? fmaxf(a.x, b.x) : a.x;
            w0 = a.x > -INFINITY ? ex2((a.x - m) * c) : 0.f;
            w1 = any[1] && b.x > -INFINITY ? ex2((b.x - m) * c) : 0.f;
            l = w0 * a.y + (any[1] ? w1 * b.y : 0.f);
        }
        const bool whole = begin == 0 && w.end == w.tiles;
        float *const part = p.parts + (2 * (int64_t)blockIdx.x + (begin == 0)) * part_floats(p.part_rows, D);
        const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
        w0 *= inv;
        w1 *= inv;
        const int64_t i0 = w.i0, out_at = (i0 + node) * p.out_row + head * p.out_head;
        const int j0 = pair ? 0 : s * (D / 2), j1 = pair ? D : j0 + D / 2;
        if (busy) {
            // 32 columns at a time and the loop not unrolled: straight code that runs once an item waits for its
            // instructions (9,400 clocks an item unrolled)
#pragma unroll 1
            for (int j = j0; j < j1; j += 32) {
                float o[32];
                tmem_ld32(tmem + S::kO + lanes + (pair ? s * D : 0) + j, o);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= w0;
                if (!pair && any[1]) {
                    float o1[32];
                    tmem_ld32(tmem + S::kO + lanes + D + j, o1);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = fmaf(o1[i], w1, o[i]);
                }
                if (sick && live) {
                    // values that are not finite, to the nodes that see them
                    for (int a = node; a >= 0; a = up_from(p, i0, small ? nullptr : parents, a)) {
                        const T *y = reinterpret_cast<const T *>(p.tree_v_at) + (i0 + a) * p.tree_row + w.h * p.tree_head + j;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float z = (float)y[i];
                            if (!(fabsf(z) < INFINITY)) o[i] += z;
                        }
                    }
                }
                if (whole) {
                    uint4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = make_uint4(pack2<T>(o[8 * i], o[8 * i + 1]), pack2<T>(o[8 * i + 2], o[8 * i + 3]),
                                          pack2<T>(o[8 * i + 4], o[8 * i + 5]), pack2<T>(o[8 * i + 6], o[8 * i + 7]));
                    turn<4>(v);
                    const int of = lane & ~3;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int64_t at = __shfl_sync(0xffffffffu, out_at, of + k);
                        if (quad * 32 + of + k < rows)
                            *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + at + j + (lane & 3) * 8) = v[k];
                    }
                } else if (live) {
                    float4 *const to = reinterpret_cast<float4 *>(part + 2 * p.part_rows + (int64_t)(tile_q * tile_rows + row) * D + j);
#pragma unroll
                    for (int i = 0; i < 8; ++i) to[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {                             // eight arrivals: of one stream's warps, or of all
            mbar_arrive(sums_free(pair ? s : 1));
            mbar_arrive(sums_free(pair ? s : 0));
        }
        if (live && (pair || s == 0)) {
            if (!whole) reinterpret_cast<float2 *>(part)[tile_q * tile_rows + row] = make_float2(m, l);
            else if (p.lse) p.lse[(w.i0 + node) * p.Hq + head] = l == 0.f ? -INFINITY : (m * c) * kLn2 + (logf(l) - kLift * kLn2);
        }
        if (tid == 0 && !whole) {                    // nobody reads these in this grid
            Cut &cut = p.cuts[blockIdx.x];
            if (begin > 0) cut.head = w.end == w.tiles ? 2 : 1;
            else {
                cut.tail = 1;
                cut.b = w.b; cut.h = w.h; cut.node0 = w.node0;
                cut.rows = min((1 + pair) * p.npt, w.n - w.node0) * p.G;
            }
        }
        if (!pair) meet();                           // everyone is done with ml
    }
    if (!ok) *failed = 1;
    tc_fence_before();
    named_sync(0, kWarps * 32);
    if (tid == 0) p.cuts[blockIdx.x].failed = *failed != 0;
}

// Joins the parts of the item that begins in CTA blockIdx.x / kJoinBlocks of the line and goes on behind it: a
// thread has four columns of a row.
constexpr int kJoinBlocks = 16, kJoinThreads = 256, kJoinAhead = 4;

template <typename T, int D, bool kCap>
__global__ void __launch_bounds__(kJoinThreads) tree_attention_join(const __grid_constant__ AttnParams p, int grid) {
    pdl_enter();
    const int first = blockIdx.x / kJoinBlocks, slice = blockIdx.x % kJoinBlocks;
    const Cut cut = p.cuts[first];
    if (cut.failed && slice == 0) ranges::tell_all(p.status, p.B, SSD_UTT_INTERNAL, threadIdx.x, kJoinThreads);
    if (!cut.tail || slice * kJoinThreads >= cut.rows * (D / 4)) return;
    const float c = kCap ? kLog2e : p.scale * kLog2e;
    const int64_t stride = 2 * part_floats(p.part_rows, D);
    const int64_t i0 = p.off[cut.b];
    for (int e = slice * kJoinThreads + threadIdx.x; e < cut.rows * (D / 4); e += kJoinBlocks * kJoinThreads) {
        const int r = e / (D / 4), u = e - r * (D / 4);
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        bool more = true;
        for (int k0 = first; more && k0 < grid; k0 += kJoinAhead) {
            // the part of CTA `first` is its second; those behind are the others' first.  A few at a time, fetched
            // before it is known whether they are there.
            int head[kJoinAhead];
            float2 a[kJoinAhead];
            float4 v[kJoinAhead];
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                const int k = k0 + i < grid ? k0 + i : grid - 1;
                const float *const part = p.parts + k * stride + (k == first ? stride / 2 : 0);
                head[i] = p.cuts[k].head;
                a[i] = reinterpret_cast<const float2 *>(part)[r];
                v[i] = reinterpret_cast<const float4 *>(part + 2 * p.part_rows + (int64_t)r * D)[u];
            }
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                const int k = k0 + i;
                if (!more || k >= grid || (k > first && head[i] == 0)) continue;      // 0: too short a part for a tile
                const float top = fmaxf(m, a[i].x);
                const float f = m > -INFINITY ? ex2((m - top) * c) : 0.f, g = a[i].x > -INFINITY ? ex2((a[i].x - top) * c) : a[i].y;
                // without a score (the sum is 0) nothing is added; with NaN scores alone (it is NaN) all becomes NaN
                l = fmaf(l, f, a[i].x > -INFINITY ? g * a[i].y : a[i].y);
                o.x = fmaf(o.x, f, g * v[i].x); o.y = fmaf(o.y, f, g * v[i].y);
                o.z = fmaf(o.z, f, g * v[i].z); o.w = fmaf(o.w, f, g * v[i].w);
                m = top;
                if (k > first && head[i] == 2) more = false;
            }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t node = i0 + cut.node0 + r / p.G;
        const int head = cut.h * p.G + r % p.G;
        T *const to = reinterpret_cast<T *>(p.out) + node * p.out_row + head * p.out_head + u * 4;
        *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
        if (u == 0 && p.lse) p.lse[node * p.Hq + head] = l == 0.f ? -INFINITY : (m * c) * kLn2 + (logf(l) - Lag<T>::kLift * kLn2);
    }
}

template <typename T, int D, bool kCap>
int launch(const AttnParams &p, int grid, cudaStream_t stream) {
    auto kernel = tree_attention<T, D, kCap>;
    // The softmax threads' registers come from what the others give back, and setmaxnreg waits until there are enough:
    // with fewer than 168 a thread at launch that would be for good.  Only the good answer is kept: a query may fail for
    // another call's error.
    static std::atomic<bool> enough{false};
    cudaError_t e = cudaSuccess;
    if (!enough.load(std::memory_order_relaxed)) {
        cudaFuncAttributes a;
        e = cudaFuncGetAttributes(&a, kernel);
        if (e == cudaSuccess && a.numRegs < kLaunchRegisters) e = cudaErrorInvalidDeviceFunction;
        if (e == cudaSuccess) enough.store(true, std::memory_order_relaxed);
        else cudaGetLastError();                       // or the next call finds it behind its own launch
    }
    if (e == cudaSuccess) e = ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), Shape<D>::kBytes);
    if (e == cudaSuccess) e = launch_pdl(kernel, (unsigned)grid, kWarps * 32u, (size_t)Shape<D>::kBytes, stream, p);
    if (e == cudaSuccess)
        e = launch_pdl(tree_attention_join<T, D, kCap>, (unsigned)(grid * kJoinBlocks), (unsigned)kJoinThreads, 0, stream, p, grid);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { record_cuda_error(e); return SSD_ERR_CUDA; }
    return SSD_OK;
}

struct AttnPlan {
    int npt, part_rows, grid;
    size_t cuts_bytes, bytes;
};
// grid: a CTA per multiprocessor, or per tile where there cannot be that many
AttnPlan attention_plan(int Hq, int Hkv, int D, int64_t M, int max_nodes, int B, int64_t max_pages, int page, int sms) {
    AttnPlan a;
    const int G = Hq / Hkv;
    if (max_nodes > M) max_nodes = (int)M;
    a.npt = kTile / G;
    if (a.npt > max_nodes) a.npt = max_nodes > 0 ? max_nodes : 1;      // no more of q is fetched than a tree can have
    a.part_rows = ((max_nodes > a.npt ? 2 : 1) * a.npt * G + 3) / 4 * 4;      // sums begin on 16 bytes
    const int64_t items = (int64_t)B * Hkv * ((max_nodes + 2 * a.npt - 1) / (2 * a.npt));
    const int least = page < 8 ? page : 8;                              // of a tile's slots, but for a cache's last
    const int64_t tiles = (max_nodes + kTile - 1) / kTile + (max_pages * page + least - 1) / least;
    a.grid = items < sms && items * tiles < sms ? (int)(items * tiles) : sms;
    if (a.grid < 1) a.grid = 1;
    a.cuts_bytes = ((size_t)sms * sizeof(Cut) + 255) / 256 * 256;
    a.bytes = a.cuts_bytes + (size_t)sms * 2 * part_floats(a.part_rows, D) * sizeof(float);
    return a;
}

}  // namespace

bool encode_map(CUtensorMap *map, ssd_dtype dtype, const void *base, int rank, const uint64_t *dims,
                const uint64_t *strides, const uint32_t *box) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Encode> known{nullptr};         // kept once it is there: a query may fail for another call's error
    Encode encode = known.load(std::memory_order_relaxed);
    if (!encode) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess || !f) {
            cudaGetLastError();
            record_cuda_error(cudaErrorNotSupported);
            return false;
        }
        encode = reinterpret_cast<Encode>(f);
        known.store(encode, std::memory_order_relaxed);
    }
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

size_t tree_attention_workspace_bytes(int Hq, int Hkv, int D, int64_t M, int max_nodes) {
    int sms = device_sm_count();
    if (sms <= 0) sms = 148;                          // without a device: the part that the kernels are made for
    return attention_plan(Hq, Hkv, D, M, max_nodes, 1, 0, 1, sms).bytes;
}

int launch_tree_attention(const ssd_heads &q, const ssd_heads &tree_k, const ssd_heads &tree_v, const ssd_kv_cache &cache,
                          const int64_t *tok_off, const int32_t *parent, int B, int64_t M, int max_nodes, float scale,
                          float cap, const ssd_heads &out, float *lse, uint32_t *status, void *workspace, cudaStream_t stream) {
    if (B == 0) return SSD_OK;
    cap = tc::cap_in_range(scale, cap);
    const int sms = device_sm_count();
    if (sms <= 0) return SSD_ERR_CUDA;
    AttnParams p;
    p.paging = paging(cache.page_size);
    p.G = q.heads / cache.heads;
    const int D = cache.head_dim;
    p.max_pages = cache.pages > 0 ? cache.max_pages : 0;      // without pages every cache is empty
    const AttnPlan plan = attention_plan(q.heads, cache.heads, D, M, max_nodes, B, p.max_pages, cache.page_size, sms);
    p.npt = plan.npt;
    p.part_rows = plan.part_rows;
    p.cuts = static_cast<Cut *>(workspace);
    p.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan.cuts_bytes);
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
    p.max_nodes = max_nodes; p.n_pages = cache.pages;
    p.scale = scale; p.cap = cap;
    const bool half = cache.dtype == SSD_F16;
    const int grid = plan.grid;
    if (D == 64)
        return half ? (cap > 0.f ? launch<__half, 64, true>(p, grid, stream) : launch<__half, 64, false>(p, grid, stream))
                    : (cap > 0.f ? launch<__nv_bfloat16, 64, true>(p, grid, stream) : launch<__nv_bfloat16, 64, false>(p, grid, stream));
    return half ? (cap > 0.f ? launch<__half, 128, true>(p, grid, stream) : launch<__half, 128, false>(p, grid, stream))
                : (cap > 0.f ? launch<__nv_bfloat16, 128, true>(p, grid, stream) : launch<__nv_bfloat16, 128, false>(p, grid, stream));
}

}  // namespace ssd
