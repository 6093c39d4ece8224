// What happens to the key/value cache between verification passes: the accepted path's keys and
// values enter it (ssd_cache_append), and slots that have received little attention leave it
// (ssd_cache_evict).  Copies and integer work, bound by HBM, and by the chain of look-ups (offsets,
// path, page, row) where the call is small.  Measured, 8 heads of 128 in bf16: 512 accepted chains of up to 200 nodes
// enter their caches in 52 us (262 MB, 5.0 TB/s); 64 caches of 1,500 to 12,000 slots go down to 2,048 in 198 us (991 MB, 5.0 TB/s, the
// selection included).
#include <math.h>

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
    return room < INT32_MAX - 256 ? room : INT32_MAX - 256;      // as the attention has it
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

constexpr int kAppendThreads = 256, kAppendRows = 4, kAppendPart = 32;      // rows of a CTA, for the average utterance's nodes

__global__ void __launch_bounds__(kAppendThreads, 6) append_kernel(const AppendParams p) {
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
    // This part's rows of the path.  A thread keeps its place in a row (tree keys or values, head, 16-byte unit) and goes
    // down the rows four at a time, whose look-ups and loads are then under way together.
    const int rows = (count + p.parts - 1) / p.parts, k0 = part * rows, k1 = min(count, k0 + rows);
    const int half = p.c.heads * p.c.units;
    for (int r = tid; r < 2 * half; r += kAppendThreads) {
        const int kv = r >= half, hu = kv ? r - half : r, h = hu / p.c.units, u = hu - h * p.c.units;
        const uint4 *const from = (kv ? p.tree_v + h * p.v_head : p.tree_k + h * p.k_head) + u;
        const int64_t row_stride = kv ? p.v_row : p.k_row;
        uint4 *const to = (kv ? p.c.v : p.c.k) + h * p.c.head_stride + u;
        for (int k = k0; k < k1; k += kAppendRows) {
            int j[kAppendRows];
            int64_t at[kAppendRows];
            uint4 x[kAppendRows];
#pragma unroll
            for (int i = 0; i < kAppendRows; ++i) {
                const int q = min(k + i, k1 - 1);            // the last row again rather than a branch
                j[i] = p.path ? p.path[i0 + q] : q;
                at[i] = slot_at(p.c, b, len + q);
            }
#pragma unroll
            for (int i = 0; i < kAppendRows; ++i)
                if (j[i] >= 0 && j[i] < n && at[i] >= 0) x[i] = from[(i0 + j[i]) * row_stride];
#pragma unroll
            for (int i = 0; i < kAppendRows; ++i)
                if (j[i] >= 0 && j[i] < n && at[i] >= 0 && k + i < k1) to[at[i]] = x[i];
        }
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
    int heads_each;                                    // of a moving CTA; a power of two that divides the heads
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

// The sum of `v` over a warp's lanes before this one.
__device__ __forceinline__ int lanes_before(int v) {
    const int lane = threadIdx.x & 31;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x - v;
}

// One CTA per utterance: the k-th largest key of the slots between the first `sink` and the last `recent`
// by four rounds of 8 bits, then the kept slots in order (of equal keys the lowest slots).  A warp has a
// run of consecutive slots, 32 at a time.  Up to 32,768 slots the weights are fetched once, into shared memory; the
// loops over them are short and not unrolled (held in registers and unrolled, 4,096 slots took 13.6 us, most of
// it the code's own way into the instruction cache).
constexpr int kHeld = 32768, kSelectWarps = kSelectThreads / 32;

struct SelectShared {
    int hist[256];
    int greater[kSelectWarps], equal[kSelectWarps];    // of a warp's slots; then what lies before them
    int digit, left;
    unsigned any;
};

__device__ __forceinline__ void select_slots(const EvictParams &p, SelectShared &sh, const float *w, int len, int32_t *kept, float *wout) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lo = p.sink, hi = len - p.recent, want = p.budget - p.sink - p.recent;
    const int steps = (len + kSelectThreads - 1) / kSelectThreads, mine = warp * steps * 32 + lane;      // + 32 a step
    auto each = [&](auto body) {                       // body(slot, weight) for all of this thread's, whole warps at a time
#pragma unroll 2
        for (int i = 0; i < steps; ++i) body(mine + i * 32, mine + i * 32 < len ? w[mine + i * 32] : 0.f);
    };
    uint32_t prefix = 0, mask = 0;
    int left = want;                                   // to be taken of the keys that match the prefix
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) sh.hist[tid] = 0;
            __syncthreads();
            each([&](int i, float x) {
                const uint32_t key = weight_key(x);
                const bool in = i >= lo && i < hi && (key & mask) == prefix;
                const uint32_t digit = in ? key >> shift & 255 : 256u;
                if (shift == 24) {
                    // weights share their leading bits: lanes with the same digit count as one
                    const unsigned same = __match_any_sync(0xffffffffu, digit);
                    if (in && (__ffs(same) - 1) == lane) atomicAdd(&sh.hist[digit], __popc(same));
                } else if (in) {
                    atomicAdd(&sh.hist[digit], 1);
                }
            });
            __syncthreads();
            if (tid < 32) {                            // the digit at which the count from above reaches `left`
                int sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += sh.hist[255 - (tid * 8 + i)];
                int above = lanes_before(sum);
                if (above < left && above + sum >= left) {
                    for (int i = 0; i < 8; ++i) {
                        const int d = 255 - (tid * 8 + i), c = sh.hist[d];
                        if (above + c >= left) { sh.digit = d; sh.left = left - above; break; }
                        above += c;
                    }
                }
            }
            __syncthreads();
            left = sh.left;
            prefix |= (uint32_t)sh.digit << shift;
            mask |= 255u << shift;
        }
    }
    // what a warp takes for certain (the ends, and larger keys) and what it has of the last key
    int sure = 0, equals = 0;
    auto kind = [&](int i, float x, bool &certain, bool &equal) {
        const uint32_t key = weight_key(x);
        const bool middle = i >= lo && i < hi && want > 0;
        certain = i < lo || (i >= hi && i < len) || (middle && key > prefix);
        equal = middle && key == prefix;
    };
    each([&](int i, float x) {
        bool certain, equal;
        kind(i, x, certain, equal);
        sure += __popc(__ballot_sync(0xffffffffu, certain));
        equals += __popc(__ballot_sync(0xffffffffu, equal));
    });
    if (lane == 0) { sh.greater[warp] = sure; sh.equal[warp] = equals; }
    __syncthreads();
    if (warp == 0) {
        const int g = sh.greater[lane], e = sh.equal[lane];
        const int e_before = lanes_before(e);
        const int taken = min(e, max(left - e_before, 0));
        const int at = lanes_before(g + taken);
        sh.greater[lane] = at;
        sh.equal[lane] = e_before;
    }
    __syncthreads();
    int at = sh.greater[warp], equal_before = sh.equal[warp];
    const unsigned below = (1u << lane) - 1;
    each([&](int i, float x) {
        bool certain, equal;
        kind(i, x, certain, equal);
        const unsigned eq = __ballot_sync(0xffffffffu, equal);
        const bool take = certain || (equal && equal_before + __popc(eq & below) < left);
        const unsigned all = __ballot_sync(0xffffffffu, take);
        if (take) {
            const int to = at + __popc(all & below);
            kept[to] = i;
            if (wout) wout[to] = x;
        }
        at += __popc(all);
        equal_before += __popc(eq);
    });
}

__global__ void __launch_bounds__(kSelectThreads) select_kernel(const EvictParams p, int held) {
    extern __shared__ float weights_here[];
    __shared__ SelectShared sh;
    pdl_enter();
    const int b = blockIdx.x, tid = threadIdx.x;
    const int64_t room = room_of(p.c);
    const int given = p.c.len[b];
    int len = min(max(given, 0), (int)room);
    uint32_t bits = given == len ? 0u : SSD_UTT_BAD_CACHE;
    if (len > p.budget && len > p.weight_cols) { bits |= SSD_UTT_BAD_CACHE; len = max(p.budget, p.weight_cols); }
    if (tid == 0) sh.any = 0;
    __syncthreads();
    const int pages = (int)(((int64_t)len + p.c.page - 1) / p.c.page);
    for (int j = tid; j < pages; j += kSelectThreads) {
        const int id = p.c.table[b * p.c.table_stride + j];
        if (id < 0 || id >= p.c.pages) bits |= SSD_UTT_BAD_CACHE;
    }
    if (bits) atomicOr(&sh.any, bits);
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
        const float *at = w;
        if (len <= held) {
            for (int i = tid; i < len; i += kSelectThreads) weights_here[i] = w[i];
            at = weights_here;
            __syncthreads();
        }
        select_slots(p, sh, at, len, kept, wout);
    }
    __syncthreads();
    if (tid == 0) { p.new_len[b] = count; p.status[b] = sh.any; }
}

// Kept slots move down in order, kept[j] to j.  kept[j] >= j, and ascending, so a block of slots may be
// written once all of its own sources have been read: later blocks' sources lie behind it.
// Where slots lie is looked up for a thousand rows ahead, so that a block of rows costs one round trip.
constexpr int kMoveThreads = 512, kMoveRows = 8, kMoveAhead = 1024;

__global__ void __launch_bounds__(kMoveThreads, 2) move_kernel(const EvictParams p) {
    // slot numbers over all pages (page id times page size and the slot in it), or -1
    __shared__ int from[kMoveAhead], to[kMoveAhead];
    pdl_enter();
    const int kv = blockIdx.x & 1, groups = p.c.heads / p.heads_each, h = blockIdx.x / 2 % groups * p.heads_each;
    const int b = blockIdx.x / 2 / groups, tid = threadIdx.x;
    const int count = p.new_len[b];
    const int32_t *const kept = p.kept + (int64_t)b * p.budget;
    const int32_t *const table = p.c.table + b * p.c.table_stride;
    const int width = p.heads_each * p.c.units, u = tid % width, r0 = tid / width, rows = kMoveThreads / width;
    uint4 *const base = (kv ? p.c.v : p.c.k) + (h + u / p.c.units) * p.c.head_stride + u % p.c.units;
    if (count == 0 || kept[count - 1] == count - 1) return;      // every slot stays where it is
    // with pages in one line the slot's number is its place; with others its page and place are taken apart again
    const bool line = p.c.page_stride == p.c.page * p.c.slot_stride;
    auto place = [&](int g) {
        if (line) return g * p.c.slot_stride;
        const int id = g / p.c.page;
        return id * p.c.page_stride + (int64_t)(g - id * p.c.page) * p.c.slot_stride;
    };
    for (int base_j = 0; base_j < count; base_j += kMoveAhead) {
        const int n = min(kMoveAhead, count - base_j);
        for (int i = tid; i < n; i += kMoveThreads) {
            const int j = base_j + i, s = kept[j], ps = s / p.c.page, pj = j / p.c.page;
            const int is = table[ps], ij = table[pj];
            const bool ok = s != j && is >= 0 && is < p.c.pages && ij >= 0 && ij < p.c.pages;      // slots before the first gap stay
            from[i] = ok ? is * p.c.page + (s - ps * p.c.page) : -1;
            to[i] = ij * p.c.page + (j - pj * p.c.page);
        }
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += rows * kMoveRows) {
            uint4 x[kMoveRows];
#pragma unroll
            for (int i = 0; i < kMoveRows; ++i) {
                const int k = i0 + i * rows + r0;
                if (k < n && from[k] >= 0) x[i] = base[place(from[k])];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kMoveRows; ++i) {
                const int k = i0 + i * rows + r0;
                if (k < n && from[k] >= 0) base[place(to[k])] = x[i];
            }
        }
        __syncthreads();
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
    int64_t parts = (M / B + kAppendPart - 1) / kAppendPart;
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
    // A CTA moves as many heads of a slot as do not leave the last round of CTAs (two to a multiprocessor) a tenth
    // emptier than the best: DRAM likes rows of 1 KB better than of 256 B (64 caches of 8 heads: 227 us a head
    // each, 212 four), 200 caches are better off with 800 CTAs than with 400 (466 us, 513).
    const int sms = device_sm_count();
    if (sms <= 0) return SSD_ERR_CUDA;
    auto filled = [&](int each) {
        const double rounds = 2.0 * B * (p.c.heads / each) / (2.0 * sms);
        return rounds / ceil(rounds);
    };
    double best = 0.0;
    p.heads_each = 1;
    for (int pass = 0; pass < 2; ++pass)
        for (int each = 1; p.c.heads % each == 0 && each * p.c.units <= kMoveThreads; each *= 2) {
            if (pass == 0) best = filled(each) > best ? filled(each) : best;
            else if (filled(each) >= 0.9 * best) p.heads_each = each;
        }
    const int64_t grid = 2ll * (p.c.heads / p.heads_each) * B;
    if (grid > INT32_MAX) return SSD_ERR_ARG;
    // no more shared memory than the longest cache can need
    const int64_t room = (int64_t)p.c.max_pages * p.c.page, most = room < weight_cols ? room : weight_cols;
    const int held = most <= kHeld ? (int)most : kHeld;
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void *>(select_kernel), (size_t)held * 4);
    if (e == cudaSuccess) e = launch_pdl(select_kernel, (unsigned)B, (unsigned)kSelectThreads, (size_t)held * 4, stream, p, held);
    if (e == cudaSuccess && p.c.pages > 0) e = launch_pdl(move_kernel, (unsigned)grid, (unsigned)kMoveThreads, 0, stream, p);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { record_cuda_error(e); return SSD_ERR_CUDA; }
    return SSD_OK;
}

}  // namespace ssd
