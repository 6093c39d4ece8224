// Attention weight that every cached slot has received (ssd_cache_weights):
//   weight[b, s] += sum over the counted nodes i of b and their heads of exp(s_is - lse_i).
//
// The scores are computed transposed, keys as the rows of the product and queries as its columns: a thread
// holds one key and adds over the columns in its registers, so nothing crosses lanes and every slot has one
// writer.  A CTA has a tile of 128 slots and goes over the heads, and over tiles of queries within a head;
// where there are few tiles, the heads are dealt out to a cluster of CTAs whose sums meet in shared memory.  Two
// groups of four warps take turns at the products' results, warp 8 issues the copies of queries, warp 10 those of
// keys, warp 9 the products.  (One warp for both kinds kept keys waiting for queries' slots: 184 us instead of 156
// on 128 caches of 500 to 3,000 slots, 896 MB.)
//
// Measured: trees of 5 to 32 nodes on 32 caches of 500 to 3,000 slots, 16 heads of 128, fp16: 48 us, 224 MB at 4.6 TB/s;
// one token's weights over 8 caches of up to 2,000 slots: 8.8 us with the host's call.
#include <float.h>
#include <math.h>

#include "ssd_tc.cuh"

namespace ssd {
namespace {

using namespace tc;

constexpr int kWarps = 11;

struct alignas(64) WeightParams {
    CUtensorMap q, cache_k;
    const int32_t *table, *len;
    const int64_t *off;
    const float *lse;
    const uint8_t *use;
    float *weight;
    uint32_t *status;
    int64_t table_stride, weight_stride, M;
    int Hq, Hkv, G, npt, q_rows, max_nodes, n_pages, max_pages, weight_cols, tiles, split;
    Paging paging;
    float scale, cap;
};

// Keys and queries have slots of their own: a head's keys stay while its tiles of queries pass, however many.
template <int D> struct WShape {
    static constexpr int kBlocks = D / 64;
    static constexpr int kKeyBytes = kBlocks * kBlockBytes, kKeySlots = D == 128 ? 2 : 4;
    static constexpr int kQueries = kKeySlots * kKeyBytes, kQueryBytes = 32768;      // two tiles, or one of more than 64 rows of 128
    static constexpr int kBars = kQueries + kQueryBytes;           // keys full[], empty[], queries full[2], empty[2], scores[2], free[2]
    static constexpr int kNumBars = 2 * kKeySlots + 8;
    static constexpr int kWords = kBars + kNumBars * 8;            // tmem address, failed
    static constexpr int kLse = (kWords + 8 + 15) / 16 * 16;       // [8][128], times log2 e: a warp's own, so that none waits
    static constexpr int kSums = kLse + 8 * kTile * 4;             // for another; [2][128]
    static constexpr int kBytes = kSums + 2 * kTile * 4;
};
// two CTAs fit a multiprocessor: one's end hides in the other's work
static_assert(2 * (WShape<128>::kBytes + 1024) <= 233472 && 2 * (WShape<64>::kBytes + 1024) <= 233472, "shared memory of two CTAs");
// Rows of a tile of queries: 64 where two such tiles take the place of one of 128.
inline int query_rows(int D, int G) { return D == 128 && G <= 64 ? 64 : kTile; }

template <typename T, int D, bool kCap>
__global__ void __launch_bounds__(kWarps * 32, 2) cache_weights(const __grid_constant__ WeightParams p) {
    using S = WShape<D>;
    extern __shared__ __align__(1024) uint8_t base[];
    const uint32_t smem = smem_u32(base);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = blockIdx.x % p.split, tile = blockIdx.x / p.split % p.tiles, b = blockIdx.x / p.split / p.tiles;
    pdl_wait();
    const int64_t i0 = p.off[b], i1 = p.off[b + 1];
    const int given = p.len[b];
    const bool rows_ok = !(i0 < 0 || i1 < i0 || i1 > p.M || i1 - i0 > p.max_nodes);
    const int n = rows_ok ? (int)(i1 - i0) : 0;
    const int64_t room = (int64_t)p.max_pages * p.paging.page;
    const int most = (int)min(min(room, (int64_t)p.weight_cols), kMostSlots);
    const int len = min(max(given, 0), most);
    if (tile == 0 && rank == 0 && warp == 0) {
        uint32_t bits = rows_ok ? 0u : SSD_UTT_BAD_OFFSETS;
        if (given != len) bits |= SSD_UTT_BAD_CACHE;
        const int pages = (int)(((int64_t)len + p.paging.page - 1) / p.paging.page);
        for (int j = lane; j < pages; j += 32) {
            const int id = p.table[b * p.table_stride + j];
            if (id < 0 || id >= p.n_pages) bits |= SSD_UTT_BAD_CACHE;
        }
        bits = __reduce_or_sync(0xffffffffu, bits);
        if (lane == 0) p.status[b] = bits;
    }
    if (n == 0 || tile >= paged_tiles(p.paging, len)) {          // the whole cluster
        pdl_launch_dependents();
        return;
    }
    const TileAt at = paged_tile(p.paging, len, tile);
    const int chunks = (n + p.npt - 1) / p.npt;
    const int heads = (p.Hkv - rank + p.split - 1) / p.split;    // of this CTA: rank, rank + split, ...
    const int units = heads * chunks;

    const int q_slots = p.q_rows * 128 * S::kBlocks * 2 <= S::kQueryBytes ? 2 : 1, q_block = p.q_rows * 128;
    const uint32_t bars = smem + S::kBars, more = bars + 16 * S::kKeySlots;
    auto keys_full = [&](int k) { return bars + 8 * (k % S::kKeySlots); };
    auto keys_empty = [&](int k) { return bars + 8 * (S::kKeySlots + k % S::kKeySlots); };
    auto q_full = [&](int i) { return more + 8 * i; };
    auto q_empty = [&](int i) { return more + 16 + 8 * i; };
    auto scores_full = [&](int s) { return more + 32 + 8 * s; };
    auto scores_free = [&](int s) { return more + 48 + 8 * s; };
    volatile uint32_t *const words = reinterpret_cast<volatile uint32_t *>(base + S::kWords);
    float *const sums = reinterpret_cast<float *>(base + S::kSums);
    auto keys_at = [&](int k) { return smem + (k % S::kKeySlots) * S::kKeyBytes; };
    auto q_at = [&](int i) { return smem + S::kQueries + i * S::kBlocks * q_block; };

    if (warp == 8) tmem_alloc(smem + S::kWords, 256);
    if (tid == 0) {
        for (int i = 0; i < S::kKeySlots; ++i) { mbar_init(keys_full(i), 1); mbar_init(keys_empty(i), 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full(s), 1);
            mbar_init(q_empty(s), 1);
            mbar_init(scores_full(s), 1);
            mbar_init(scores_free(s), 4);
        }
        mbar_init_fence();
        words[1] = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = words[0];

    if (warp == 10) {
        const int page_count = p.paging.pages ? p.paging.pages : 1;
        int id = p.n_pages;                                      // outside: the copy fills in zeros
        if (lane < page_count && at.page + lane < p.max_pages) {
            id = p.table[b * p.table_stride + at.page + lane];
            if (id < 0 || id >= p.n_pages) id = p.n_pages;
        }
        const int box = p.paging.box, copies = (at.valid + box - 1) / box;
        // copies are of 64 columns and 8 rows at least: a lane for each
        const int i = lane / S::kBlocks, x = lane % S::kBlocks;
        const int page = __shfl_sync(0xffffffffu, id, p.paging.pages ? i : 0);
        bool ok = true;
        for (int k = 0; k < heads && ok; ++k) {
            if (k >= S::kKeySlots) ok = mbar_wait_bounded(keys_empty(k), (k / S::kKeySlots - 1) & 1);
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(keys_full(k), copies * box * 128 * S::kBlocks);
            __syncwarp();
            if (i < copies)
                tma_load_4d(keys_at(k) + x * kBlockBytes + i * box * 128, &p.cache_k, x * 64, rank + k * p.split,
                            p.paging.pages ? 0 : at.slot + i * box, page, keys_full(k));
        }
        if (!ok) words[1] = 1;
    } else if (warp == 8) {
        bool ok = true;
        for (int k = 0, u = 0; k < heads && ok; ++k) {
            for (int c = 0; c < chunks && ok; ++c, ++u) {
                const int q = u % q_slots;
                if (u >= q_slots) ok = mbar_wait_bounded(q_empty(q), (u / q_slots - 1) & 1);
                if (!ok) break;
                if (lane == 0) mbar_arrive_expect_tx(q_full(q), p.G * p.npt * 128 * S::kBlocks);
                __syncwarp();
                if (lane < S::kBlocks)
                    tma_load_3d(q_at(q) + lane * q_block, &p.q, lane * 64, (rank + k * p.split) * p.G, (int)i0 + c * p.npt, q_full(q));
            }
        }
        if (!ok) words[1] = 1;
    } else if (warp == 9) {
        bool ok = true;
        const uint32_t tm = uniform(tmem);
        for (int u = 0; u < units && ok; ++u) {
            const int k = u / chunks, c = u - k * chunks, s = u & 1, q = u % q_slots;
            ok = mbar_wait_bounded(keys_full(k), (k / S::kKeySlots) & 1) && mbar_wait_bounded(q_full(q), (u / q_slots) & 1);
            if (u > 1) ok = ok && mbar_wait_bounded(scores_free(s), ((u >> 1) - 1) & 1);
            if (!ok) break;
            tc_fence_after();
            const int rows = uniform(min(p.npt, n - c * p.npt) * p.G);
            if (elect_one()) {
                const uint32_t idesc = instruction<T>((rows + 15) / 16 * 16, false);
                const uint64_t a = operand(keys_at(k)), b = operand(q_at(q));
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
                    mma_ss(tm + s * kTile, a + (x >> 2) * (kBlockBytes >> 4) + (x & 3) * 2, b + (x >> 2) * (q_block >> 4) + (x & 3) * 2,
                           idesc, x > 0);
                mma_commit(scores_full(s));
                mma_commit(q_empty(q));
                if (c == chunks - 1) mma_commit(keys_empty(k));
            }
            __syncwarp();
        }
        if (!ok) words[1] = 1;
    } else {
        const int s = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t t_scores = tmem + s * kTile + ((uint32_t)((warp & 3) * 32) << 16);
        float *const lse = reinterpret_cast<float *>(base + S::kLse) + warp * kTile;
        const bool busy = (warp & 3) * 32 < at.valid;
        const float c = kCap ? kLog2e : p.scale * kLog2e;
        float sum = 0.f;
        bool ok = true;
        for (int u = s; u < units; u += 2) {
            const int chunk = u % chunks, h = rank + u / chunks * p.split, k = u >> 1;
            const int rows = min(p.npt, n - chunk * p.npt) * p.G;
            if (busy) {
                __syncwarp();                                    // the last unit's are read
                for (int r = lane; r < (rows + 15) / 16 * 16; r += 32) {
                    float x = INFINITY;                          // not counted: the probability is 0
                    const int64_t node = i0 + chunk * p.npt + r / p.G;
                    if (r < rows && (!p.use || p.use[node])) {
                        x = p.lse[node * p.Hq + h * p.G + r % p.G] * kLog2e;
                        if (x == INFINITY) x = FLT_MAX;          // a counted row's infinity: 0 all the same, but for a score of NaN
                    }
                    lse[r] = x;
                }
                __syncwarp();
            }
            ok = mbar_wait_bounded(scores_full(s), k & 1);
            if (!ok) break;
            tc_fence_after();
            if (busy) {
                for (int j = 0; j < rows; j += 32) {
                    float x[32], a[4] = {0.f, 0.f, 0.f, 0.f};
                    const bool half = rows - j <= 16;            // the product wrote no more than that
                    if (half) tmem_ld16(t_scores + j, x); else tmem_ld32(t_scores + j, x);
                    tmem_wait_ld();
                    if (kCap) { if (half) cap_scores<16>(x, p.scale, p.cap, row < at.valid); else cap_scores<32>(x, p.scale, p.cap, row < at.valid); }
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (i >= 16 && half) break;
                        x[i] = ex2(fmaf(x[i], c, -lse[j + i]));
                        a[i & 3] += x[i];
                    }
                    float more = (a[0] + a[1]) + (a[2] + a[3]);
                    if (more != more) {                          // a NaN: of a row that counts, or of one that does not
                        a[0] = a[1] = a[2] = a[3] = 0.f;         // (added in the same order: the same bits without it)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < 16 || !half) a[i & 3] += lse[j + i] == INFINITY ? 0.f : x[i];
                        more = (a[0] + a[1]) + (a[2] + a[3]);
                    }
                    sum += more;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(scores_free(s));
        }
        if (!ok) words[1] = 1;
        sums[s * kTile + row] = sum;
    }
    __syncthreads();
    if (p.split > 1) { cluster_arrive(); cluster_wait(); }
    if (rank == 0 && tid < at.valid) {
        float sum = 0.f;
        for (int k = 0; k < p.split; ++k)
            for (int s = 0; s < 2; ++s) {
                const uint32_t a = smem + S::kSums + (s * kTile + tid) * 4;
                float v;
                if (p.split > 1) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_address(a, k)) : "memory");
                else v = sums[s * kTile + tid];
                sum += v;
            }
        const int slot = at.page * p.paging.page + at.slot + tid;
        p.weight[b * p.weight_stride + slot] += sum;
    }
    if (p.split > 1) { cluster_arrive(); cluster_wait(); }
    if (words[1]) {
        drain_after_error();
        if (tid == 0) p.status[b] = SSD_UTT_INTERNAL;
    }
    __syncthreads();
    if (warp == 8) { tc_fence_after(); tmem_free(tmem, 256); }
}

template <typename T, int D, bool kCap> int launch(const WeightParams &p, int64_t grid, cudaStream_t stream) {
    auto kernel = cache_weights<T, D, kCap>;
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), WShape<D>::kBytes);
    if (e == cudaSuccess)
        e = launch_clusters(kernel, (unsigned)p.split, (unsigned)grid, kWarps * 32u, (size_t)WShape<D>::kBytes, stream, p);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { record_cuda_error(e); return SSD_ERR_CUDA; }
    return SSD_OK;
}

}  // namespace

int launch_cache_weights(const ssd_heads &q, const float *lse, const ssd_kv_cache &cache, const int64_t *tok_off, int B,
                         int64_t M, int max_nodes, float scale, float cap, const uint8_t *use, float *weight,
                         int64_t weight_stride, int weight_cols, uint32_t *status, cudaStream_t stream) {
    if (B == 0) return SSD_OK;
    cap = tc::cap_in_range(scale, cap);
    WeightParams p;
    p.paging = paging(cache.page_size);
    p.G = q.heads / cache.heads;
    p.q_rows = query_rows(cache.head_dim, p.G);
    p.npt = p.q_rows / p.G;
    if (p.npt > max_nodes) p.npt = max_nodes > 0 ? max_nodes : 1;
    const int D = cache.head_dim;
    if (M > 0 && !encode_rows(&p.q, cache.dtype, q, D, M, p.G, p.npt)) return SSD_ERR_CUDA;
    if (cache.pages > 0 && !encode_cache(&p.cache_k, cache, cache.k, p.paging.box)) return SSD_ERR_CUDA;
    p.table = cache.page_table; p.len = cache.len; p.off = tok_off; p.lse = lse; p.use = use;
    p.weight = weight; p.status = status; p.table_stride = cache.table_stride; p.weight_stride = weight_stride; p.M = M;
    p.Hq = q.heads; p.Hkv = cache.heads; p.max_nodes = max_nodes; p.n_pages = cache.pages;
    p.max_pages = cache.pages > 0 ? cache.max_pages : 0;
    p.weight_cols = weight_cols; p.scale = scale; p.cap = cap;
    const int sms = device_sm_count();
    if (sms <= 0) return SSD_ERR_CUDA;
    int64_t room = (int64_t)p.max_pages * cache.page_size;
    if (room > weight_cols) room = weight_cols;
    const int64_t tiles = paged_tiles(p.paging, (int)(room < kMostSlots ? room : kMostSlots));
    p.tiles = tiles > 0 ? (int)tiles : 1;
    p.split = 1;
    while (p.split < 8 && p.split * 2 <= p.Hkv && (int64_t)B * p.tiles * p.split * 2 <= 2 * sms) p.split *= 2;
    const int64_t grid = (int64_t)B * p.tiles * p.split;
    if (grid > INT32_MAX) return SSD_ERR_ARG;
    const bool half = cache.dtype == SSD_F16;
    if (D == 64)
        return half ? (cap > 0.f ? launch<__half, 64, true>(p, grid, stream) : launch<__half, 64, false>(p, grid, stream))
                    : (cap > 0.f ? launch<__nv_bfloat16, 64, true>(p, grid, stream) : launch<__nv_bfloat16, 64, false>(p, grid, stream));
    return half ? (cap > 0.f ? launch<__half, 128, true>(p, grid, stream) : launch<__half, 128, false>(p, grid, stream))
                : (cap > 0.f ? launch<__nv_bfloat16, 128, true>(p, grid, stream) : launch<__nv_bfloat16, 128, false>(p, grid, stream));
}

}  // namespace ssd
