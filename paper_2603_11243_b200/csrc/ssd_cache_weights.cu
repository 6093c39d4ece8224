// Attention weight that every cached slot has received (ssd_cache_weights):
//   weight[b, s] += sum over the counted nodes i of b and their heads of exp(s_is - lse_i).
//
// The scores are computed transposed, keys as the rows of the product and queries as its columns: a thread
// holds one key and adds over the columns in its registers, so nothing crosses lanes and every slot has one
// writer.  A CTA has a tile of 128 slots and goes over the heads, and over tiles of queries within a head;
// where there are few tiles, the heads are dealt out to a cluster of CTAs whose sums meet in shared memory.  Two
// groups of four warps take turns at the products' results, warp 8 issues the copies, warp 9 the products.
#include <math.h>

#include "ssd_tc.cuh"

namespace ssd {
namespace {

using namespace tc;

constexpr int kWarps = 10;

struct alignas(64) WeightParams {
    CUtensorMap q, cache_k;
    const int32_t *table, *len;
    const int64_t *off;
    const float *lse;
    const uint8_t *use;
    float *weight;
    uint32_t *status;
    int64_t table_stride, weight_stride, M;
    int Hq, Hkv, G, npt, max_nodes, n_pages, max_pages, weight_cols, tiles, split;
    Paging paging;
    float scale, cap;
};

template <int D> struct WShape {
    static constexpr int kBlocks = D / 64;
    static constexpr int kSlotBytes = kBlocks * kBlockBytes;
    static constexpr int kSlots = D == 128 ? 3 : 6;                // two CTAs fit a multiprocessor: one's end hides in the other's work
    static constexpr int kBars = kSlots * kSlotBytes;              // full[], empty[], scores[2], free[2]
    static constexpr int kNumBars = 2 * kSlots + 4;
    static constexpr int kWords = kBars + kNumBars * 8;            // tmem address, failed
    static constexpr int kLse = (kWords + 8 + 15) / 16 * 16;       // [2][128], times log2 e
    static constexpr int kSums = kLse + 2 * kTile * 4;             // [2][128]
    static constexpr int kBytes = kSums + 2 * kTile * 4;
};
static_assert(2 * (WShape<128>::kBytes + 1024) <= 233472 && 2 * (WShape<64>::kBytes + 1024) <= 233472, "shared memory of two CTAs");

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
    const int most = (int)min(min(room, (int64_t)p.weight_cols), (int64_t)INT32_MAX);
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

    auto full = [&](int i) { return smem + S::kBars + 8 * i; };
    auto empty = [&](int i) { return smem + S::kBars + 8 * (S::kSlots + i); };
    auto scores_full = [&](int s) { return smem + S::kBars + 8 * (2 * S::kSlots + s); };
    auto scores_free = [&](int s) { return smem + S::kBars + 8 * (2 * S::kSlots + 2 + s); };
    volatile uint32_t *const words = reinterpret_cast<volatile uint32_t *>(base + S::kWords);
    float *const sums = reinterpret_cast<float *>(base + S::kSums);
    auto slot_at = [&](int pos) { return smem + (pos % S::kSlots) * S::kSlotBytes; };

    if (warp == 8) tmem_alloc(smem + S::kWords, 256);
    if (tid == 0) {
        for (int i = 0; i < S::kSlots; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(scores_full(s), 1); mbar_init(scores_free(s), 4); }
        mbar_init_fence();
        words[1] = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = words[0];

    if (warp == 8) {
        // a head's keys, then its tiles of queries
        const int page_count = p.paging.pages ? p.paging.pages : 1;
        int id = p.n_pages;                                      // outside: the copy fills in zeros
        if (lane < page_count && at.page + lane < p.max_pages) {
            id = p.table[b * p.table_stride + at.page + lane];
            if (id < 0 || id >= p.n_pages) id = p.n_pages;
        }
        const int box = p.paging.box, copies = (at.valid + box - 1) / box;
        bool ok = true;
        int pos = 0;
        auto take = [&](int bytes) {
            if (pos >= S::kSlots) ok = mbar_wait_bounded(empty(pos % S::kSlots), (pos / S::kSlots - 1) & 1);
            if (ok && lane == 0) mbar_arrive_expect_tx(full(pos % S::kSlots), bytes);
            __syncwarp();
            return ok;
        };
        for (int k = 0; k < heads && ok; ++k) {
            const int h = rank + k * p.split;
            if (!take(copies * box * 128 * S::kBlocks)) break;
            {
                // copies are of 64 columns and 8 rows at least: a lane for each
                const int i = lane / S::kBlocks, x = lane % S::kBlocks;
                const int page = __shfl_sync(0xffffffffu, id, p.paging.pages ? i : 0);
                if (i < copies)
                    tma_load_4d(slot_at(pos) + x * kBlockBytes + i * box * 128, &p.cache_k, x * 64, h,
                                p.paging.pages ? 0 : at.slot + i * box, page, full(pos % S::kSlots));
            }
            ++pos;
            for (int c = 0; c < chunks; ++c, ++pos) {
                if (!take(p.G * p.npt * 128 * S::kBlocks)) break;
                if (lane < S::kBlocks)
                    tma_load_3d(slot_at(pos) + lane * kBlockBytes, &p.q, lane * 64, h * p.G, (int)i0 + c * p.npt, full(pos % S::kSlots));
            }
        }
        if (!ok) words[1] = 1;
    } else if (warp == 9) {
        bool ok = true;
        const uint32_t tm = uniform(tmem);
        for (int u = 0; u < units && ok; ++u) {
            const int c = u % chunks, s = u & 1, k = u >> 1;
            const int keys = u / chunks * (chunks + 1), q_pos = keys + 1 + c;
            ok = mbar_wait_bounded(full(keys % S::kSlots), (keys / S::kSlots) & 1) &&
                 mbar_wait_bounded(full(q_pos % S::kSlots), (q_pos / S::kSlots) & 1);
            if (k > 0) ok = ok && mbar_wait_bounded(scores_free(s), (k - 1) & 1);
            if (!ok) break;
            tc_fence_after();
            const int rows = uniform(min(p.npt, n - c * p.npt) * p.G);
            if (elect_one()) {
                const uint32_t idesc = instruction<T>((rows + 15) / 16 * 16, false);
                const uint64_t a = operand(slot_at(keys)), q = operand(slot_at(q_pos));
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const int o = (x >> 2) * (kBlockBytes >> 4) + (x & 3) * 2;
                    mma_ss(tm + s * kTile, a + o, q + o, idesc, x > 0);
                }
                mma_commit(scores_full(s));
                mma_commit(empty(q_pos % S::kSlots));
                if (c == chunks - 1) mma_commit(empty(keys % S::kSlots));
            }
            __syncwarp();
        }
        if (!ok) words[1] = 1;
    } else {
        const int s = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t t_scores = tmem + s * kTile + ((uint32_t)((warp & 3) * 32) << 16);
        float *const lse = reinterpret_cast<float *>(base + S::kLse) + s * kTile;
        const bool busy = (warp & 3) * 32 < at.valid;
        const float c = kCap ? kLog2e : p.scale * kLog2e;
        float sum = 0.f;
        bool ok = true;
        for (int u = s; u < units; u += 2) {
            const int chunk = u % chunks, h = rank + u / chunks * p.split, k = u >> 1;
            const int rows = min(p.npt, n - chunk * p.npt) * p.G;
            named_sync(1 + s, 128);                              // everyone is done with the last unit's
            {
                const int64_t node = i0 + chunk * p.npt + row / p.G;
                float x = INFINITY;                              // not counted: the probability is 0
                if (row < rows && (!p.use || p.use[node])) x = p.lse[node * p.Hq + h * p.G + row % p.G] * kLog2e;
                lse[row] = x;
            }
            named_sync(1 + s, 128);
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
                            if (i < 16 || !half) a[i & 3] += lse[j + i] < INFINITY ? x[i] : 0.f;
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
    WeightParams p;
    p.paging = paging(cache.page_size);
    p.G = q.heads / cache.heads;
    p.npt = kTile / p.G;
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
    const int64_t tiles = paged_tiles(p.paging, (int)(room < INT32_MAX - 2 * kTile ? room : INT32_MAX - 2 * kTile));
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
