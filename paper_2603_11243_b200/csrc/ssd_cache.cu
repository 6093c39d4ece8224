// What happens to the key/value cache between verification passes: the accepted path's keys and
// values enter it (ssd_cache_append), and slots that have received little attention leave it
// (ssd_cache_evict).  Copies and integer work, bound by HBM, and by the chain of look-ups (offsets,
// path, page, row) where the call is small.
#include "ssd_common.cuh"

namespace ssd {
namespace {

struct CacheParams {
    uint4 *k, *v;
    int64_t page_stride, slot_stride, head_stride;     // in units of 16 bytes
    const int32_t *table, *len;
    int64_t table_stride;
    int pages, page, heads, units, max_pages;          // units: of 16 bytes in a head
};
CacheParams cache_params(const ssd_kv_cache &c) {
    CacheParams p;
    p.k = static_cast<uint4 *>(c.k); p.v = static_cast<uint4 *>(c.v);
    p.page_stride = c.page_stride / 8; p.slot_stride = c.slot_stride / 8; p.head_stride = c.head_stride / 8;
    p.table = c.page_table; p.len = c.len; p.table_stride = c.table_stride;
    p.pages = c.pages; p.page = c.page_size; p.heads = c.heads; p.units = c.head_dim / 8;
    p.max_pages = c.pages > 0 ? c.max_pages : 0;
    return p;
}
__device__ __forceinline__ int64_t room_of(const CacheParams &c) {
    const int64_t room = (int64_t)c.max_pages * c.page;
    return room < INT32_MAX ? room : INT32_MAX;
}
// Where slot s of utterance b lies, in units from the cache's base; -1: its page is none of the cache's.
__device__ __forceinline__ int64_t slot_at(const CacheParams &c, int b, int s) {
    const int pg = s / c.page;
    const int id = c.table[b * c.table_stride + pg];
    if (id < 0 || id >= c.pages) return -1;
    return id * c.page_stride + (int64_t)(s - pg * c.page) * c.slot_stride;
}

// ---- append ----------------------------------------------------------------------------------------
struct AppendParams {
    CacheParams c;
    const uint4 *tree_k, *tree_v;
    int64_t k_row, k_head, v_row, v_head;              // in units of 16 bytes
    const int64_t *off;
    const int32_t *path, *path_len;
    float *weight;
    int64_t weight_stride, M;
    int weight_cols, parts;
    int32_t *new_len;
    uint32_t *status;
};

constexpr int kAppendThreads = 256;

__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendParams p) {
    pdl_enter();
    const int b = blockIdx.x / p.parts, part = blockIdx.x % p.parts, tid = threadIdx.x;
    const int64_t i0 = p.off[b], i1 = p.off[b + 1];
    const int len = p.c.len[b], take = p.path_len[b];
    const bool rows_ok = !(i0 < 0 || i1 < i0 || i1 > p.M);
    const int n = rows_ok ? (int)min(i1 - i0, (int64_t)INT32_MAX) : 0;
    const int64_t room = room_of(p.c);
    uint32_t bits = 0;
    if (!rows_ok) bits |= SSD_UTT_BAD_OFFSETS;
    if (len < 0 || len > room) bits |= SSD_UTT_BAD_CACHE;
    if (take < 0 || (rows_ok && take > n)) bits |= SSD_UTT_BAD_PARENT;
    if (!bits && len + (int64_t)take > room) bits |= SSD_UTT_CACHE_FULL;
    const int count = bits ? 0 : take;
    const int per_row = 2 * p.c.heads * p.c.units, step = p.parts * kAppendThreads;
    const int64_t all = (int64_t)count * per_row;
    for (int64_t e = (int64_t)part * kAppendThreads + tid; e < all; e += step) {
        const int k = (int)(e / per_row), r = (int)(e - (int64_t)k * per_row);
        const int kv = r >= p.c.heads * p.c.units, hu = kv ? r - p.c.heads * p.c.units : r;
        const int h = hu / p.c.units, u = hu - h * p.c.units;
        const int j = p.path ? p.path[i0 + k] : k;
        const int64_t at = slot_at(p.c, b, len + k);
        if (j < 0 || j >= n || at < 0) continue;
        const uint4 *from = kv ? p.tree_v + (i0 + j) * p.v_row + h * p.v_head : p.tree_k + (i0 + j) * p.k_row + h * p.k_head;
        (kv ? p.c.v : p.c.k)[at + h * p.c.head_stride + u] = from[u];
    }
    if (part == 0) {
        for (int k = tid; k < count; k += kAppendThreads) {
            const int j = p.path ? p.path[i0 + k] : k;
            if (j < 0 || j >= n) bits |= SSD_UTT_BAD_PARENT;
            if (slot_at(p.c, b, len + k) < 0) bits |= SSD_UTT_BAD_CACHE;
            if (p.weight && len + k < p.weight_cols) p.weight[b * p.weight_stride + len + k] = 0.f;
        }
        __shared__ unsigned any;
        if (tid == 0) any = 0;
        __syncthreads();
        if (bits) atomicOr(&any, bits);
        __syncthreads();
        if (tid == 0) { p.new_len[b] = len + count; p.status[b] = any; }
    }
}

// ---- evict -----------------------------------------------------------------------------------------
struct EvictParams {
    CacheParams c;
    const float *weight;
    int64_t weight_stride;
    int weight_cols, budget, sink, recent;
    int32_t *kept;
    float *weight_out;
    int64_t out_stride;
    int32_t *new_len;
    uint32_t *status;
};

// Larger weight, larger key; -0 is 0 and NaN lies below everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelectThreads = 1024;

// Exclusive sum of `v` over the block in thread order, and the block's total.
__device__ __forceinline__ int block_scan(int v, int *warp_sums, int &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int s = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        warp_sums[lane] = s;
    }
    __syncthreads();
    const int before = warp ? warp_sums[warp - 1] : 0;
    total = warp_sums[31];
    __syncthreads();
    return before + x - v;
}

// One CTA per utterance: the k-th largest key of the slots between the first `sink` and the last `recent`
// by four rounds of 8 bits, then the kept slots in order (of equal keys the lowest slots).
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const EvictParams p) {
    __shared__ int hist[256], warp_sums[32];
    __shared__ int s_digit, s_left;
    __shared__ unsigned any;
    pdl_enter();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int64_t room = room_of(p.c);
    const int given = p.c.len[b];
    int len = min(max(given, 0), (int)room);
    uint32_t bits = given == len ? 0u : SSD_UTT_BAD_CACHE;
    if (len > p.budget && len > p.weight_cols) { bits |= SSD_UTT_BAD_CACHE; len = p.weight_cols; }
    if (tid == 0) any = 0;
    __syncthreads();
    const int pages = (int)(((int64_t)len + p.c.page - 1) / p.c.page);
    for (int j = tid; j < pages; j += kSelectThreads) {
        const int id = p.c.table[b * p.c.table_stride + j];
        if (id < 0 || id >= p.c.pages) bits |= SSD_UTT_BAD_CACHE;
    }
    if (bits) atomicOr(&any, bits);
    const float *const w = p.weight + b * p.weight_stride;
    int32_t *const kept = p.kept + (int64_t)b * p.budget;
    float *const wout = p.weight_out ? p.weight_out + b * p.out_stride : nullptr;
    const int count = min(len, p.budget);
    for (int j = count + tid; j < p.budget; j += kSelectThreads) {
        kept[j] = -1;
        if (wout) wout[j] = 0.f;
    }
    if (len <= p.budget) {
        for (int j = tid; j < len; j += kSelectThreads) {
            kept[j] = j;
            if (wout) wout[j] = j < p.weight_cols ? w[j] : 0.f;
        }
    } else {
        const int lo = p.sink, hi = len - p.recent, want = p.budget - p.sink - p.recent;
        uint32_t prefix = 0, mask = 0;
        int left = want;                               // to be taken of the keys that match the prefix
        if (want > 0) {
            for (int shift = 24; shift >= 0; shift -= 8) {
                for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0;
                __syncthreads();
                for (int i = lo + tid; i < hi; i += kSelectThreads) {
                    const uint32_t key = weight_key(w[i]);
                    if ((key & mask) == prefix) atomicAdd(&hist[key >> shift & 255], 1);
                }
                __syncthreads();
                if (tid < 32) {                        // the digit at which the count from above reaches `left`
                    int sum = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += hist[255 - (tid * 8 + i)];
                    int x = sum;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int y = __shfl_up_sync(0xffffffffu, x, o);
                        if (tid >= o) x += y;
                    }
                    int above = x - sum;
                    if (above < left && x >= left) {
                        for (int i = 0; i < 8; ++i) {
                            const int d = 255 - (tid * 8 + i), c = hist[d];
                            if (above + c >= left) { s_digit = d; s_left = left - above; break; }
                            above += c;
                        }
                    }
                }
                __syncthreads();
                left = s_left;
                prefix |= (uint32_t)s_digit << shift;
                mask |= 255u << shift;
                __syncthreads();
            }
        }
        int at = 0, equal_before = 0;
        for (int base = 0; base < len; base += kSelectThreads) {
            const int i = base + tid;
            const float x = i < len ? w[i] : 0.f;
            const uint32_t key = weight_key(x);
            const bool forced = i < lo || (i >= hi && i < len), middle = i >= lo && i < hi && want > 0;
            const bool equal = middle && key == prefix;
            int equals, total;
            const int rank = block_scan(equal, warp_sums, equals);
            const bool take = forced || (middle && key > prefix) || (equal && equal_before + rank < left);
            const int to = at + block_scan(take, warp_sums, total);
            if (take) {
                kept[to] = i;
                if (wout) wout[to] = x;
            }
            at += total;
            equal_before += equals;
        }
    }
    __syncthreads();
    if (tid == 0) { p.new_len[b] = count; p.status[b] = any; }
}

// Kept slots move down in order, kept[j] to j.  kept[j] >= j, and ascending, so a block of slots may be
// written once all of its own sources have been read: later blocks' sources lie behind it.
constexpr int kMoveThreads = 512, kMoveRows = 8;

__global__ void __launch_bounds__(kMoveThreads) move_kernel(const EvictParams p) {
    pdl_enter();
    const int kv = blockIdx.x & 1, h = blockIdx.x / 2 % p.c.heads, b = blockIdx.x / 2 / p.c.heads, tid = threadIdx.x;
    const int count = p.new_len[b];
    const int32_t *const kept = p.kept + (int64_t)b * p.budget;
    uint4 *const base = (kv ? p.c.v : p.c.k) + h * p.c.head_stride;
    const int u = tid % p.c.units, r0 = tid / p.c.units, rows = kMoveThreads / p.c.units;
    // slots before the first gap stay: kept[j] == j holds up to there and nowhere behind
    int first = 0, end = count;
    while (first < end) {
        const int mid = (first + end) >> 1;
        if (kept[mid] == mid) first = mid + 1; else end = mid;
    }
    for (int j0 = first; j0 < count; j0 += rows * kMoveRows) {
        uint4 x[kMoveRows];
        int64_t to[kMoveRows];
#pragma unroll
        for (int i = 0; i < kMoveRows; ++i) {
            const int j = j0 + i * rows + r0;
            to[i] = -1;
            if (j < count) {
                const int64_t from = slot_at(p.c, b, kept[j]);
                to[i] = from < 0 ? -1 : slot_at(p.c, b, j);
                if (to[i] >= 0) x[i] = base[from + u];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveRows; ++i)
            if (to[i] >= 0) base[to[i] + u] = x[i];
    }
}

}  // namespace

int launch_cache_append(const ssd_heads &tree_k, const ssd_heads &tree_v, const ssd_kv_cache &cache, const int64_t *tok_off,
                        const int32_t *path, const int32_t *path_len, int B, int64_t M, float *weight,
                        int64_t weight_stride, int weight_cols, int32_t *new_len, uint32_t *status, cudaStream_t stream) {
    if (B == 0) return SSD_OK;
    AppendParams p;
    p.c = cache_params(cache);
    p.tree_k = static_cast<const uint4 *>(tree_k.data); p.tree_v = static_cast<const uint4 *>(tree_v.data);
    p.k_row = tree_k.row_stride / 8; p.k_head = tree_k.head_stride / 8;
    p.v_row = tree_v.row_stride / 8; p.v_head = tree_v.head_stride / 8;
    p.off = tok_off; p.path = path; p.path_len = path_len;
    p.weight = weight; p.weight_stride = weight_stride; p.weight_cols = weight ? weight_cols : 0;
    p.M = M; p.new_len = new_len; p.status = status;
    // four units of a row a thread, for the average utterance
    const int64_t units = (M / B + 1) * 2 * p.c.heads * p.c.units;
    int64_t parts = (units + 4 * kAppendThreads - 1) / (4 * kAppendThreads);
    const int sms = device_sm_count();
    if (sms <= 0) return SSD_ERR_CUDA;
    const int64_t most = (int64_t)sms * 64 / B;
    if (parts > most) parts = most;
    p.parts = parts < 1 ? 1 : (int)parts;
    const int64_t grid = (int64_t)B * p.parts;
    if (grid > INT32_MAX) return SSD_ERR_ARG;
    cudaError_t e = launch_pdl(append_kernel, (unsigned)grid, (unsigned)kAppendThreads, 0, stream, p);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { record_cuda_error(e); return SSD_ERR_CUDA; }
    return SSD_OK;
}

int launch_cache_evict(const ssd_kv_cache &cache, const float *weight, int64_t weight_stride, int weight_cols, int B, int budget,
                       int sink, int recent, int32_t *kept, float *weight_out, int64_t out_stride, int32_t *new_len,
                       uint32_t *status, cudaStream_t stream) {
    if (B == 0) return SSD_OK;
    EvictParams p;
    p.c = cache_params(cache);
    p.weight = weight; p.weight_stride = weight_stride; p.weight_cols = weight_cols;
    p.budget = budget; p.sink = sink; p.recent = recent;
    p.kept = kept; p.weight_out = weight_out; p.out_stride = out_stride; p.new_len = new_len; p.status = status;
    const int64_t grid = 2ll * p.c.heads * B;
    if (grid > INT32_MAX) return SSD_ERR_ARG;
    cudaError_t e = launch_pdl(select_kernel, (unsigned)B, (unsigned)kSelectThreads, 0, stream, p);
    if (e == cudaSuccess && p.c.pages > 0) e = launch_pdl(move_kernel, (unsigned)grid, (unsigned)kMoveThreads, 0, stream, p);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { record_cuda_error(e); return SSD_ERR_CUDA; }
    return SSD_OK;
}

}  // namespace ssd
