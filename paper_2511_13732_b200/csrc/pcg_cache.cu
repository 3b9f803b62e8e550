// The paged key/value cache of a decoding round: the plan of the next round (lengths, block tables, slots, positions)
// and the writes of new keys and values.
#include "pcg_cache.cuh"

namespace pcg {

// ---------------------------------------------------------------------------------------------- plan
constexpr int kPlanThreads = 512;
constexpr int kPlanMaxB = 16384;

struct PlanArgs {
    int32_t B, block_size, max_blocks, ring_size, rows;
    const int32_t *cached_len, *accept_len, *new_len, *held, *ring_state;
    int32_t *block_table, *free_ring;
    int32_t *out_cached_len, *out_kv_len, *out_held, *out_row_start, *out_slots, *out_positions, *out_ring_state, *out_flags;
};

struct PlanSeq {
    bool done;
    int64_t base;  // tokens that stay cached
    int32_t n, held;
    int64_t blocks;  // blocks that base + n tokens need
};

__device__ __forceinline__ PlanSeq plan_load(const PlanArgs &a, int b) {
    PlanSeq s;
    const int32_t n = a.new_len[b];
    s.done = n < 0;
    s.n = max(n, 0);
    s.held = min(max(a.held[b], 0), a.max_blocks);
    s.base = s.done ? 0 : max((int64_t)a.cached_len[b] + (a.accept_len ? (int64_t)a.accept_len[b] + 1 : 0), (int64_t)0);
    s.blocks = (s.base + s.n + a.block_size - 1) / a.block_size;
    return s;
}

// Exclusive prefix of one int64 per thread in thread order, and the total.
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t *scratch, int64_t *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = inc;
    __syncthreads();
    int64_t base = 0, tot = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w == warp) base = tot;
        tot += scratch[w];
    }
    *total = tot;
    return base + inc - v;
}

// Every block forms the prefix sums over all sequences for itself (12 to 20 bytes a sequence, out of L2): that costs
// less than a second launch or a grid-wide exchange for any batch a server runs, and the blocks then share the rows,
// the table entries and the released blocks among themselves.  Thread t owns a contiguous run of sequences.
// What bounds it: latency -- a launch, two dependent rounds of loads and two block scans (5.3 us for one sequence, 8.2 for
// 256, 13.5 for 3001).
__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(const __grid_constant__ PlanArgs a) {
    extern __shared__ int32_t plan_smem[];
    int32_t *row_start = plan_smem;            // [B + 1], clamped to rows
    int32_t *offset = plan_smem + a.B + 1;     // [B] first ring entry of its new blocks, or of its released ones
    uint8_t *flag = (uint8_t *)(offset + a.B);  // [B]
    __shared__ int64_t scratch[kPlanThreads / 32];
    const int tid = threadIdx.x, B = a.B;
    const int per = (B + kPlanThreads - 1) / kPlanThreads, lo = min(B, tid * per), hi = min(B, lo + per);
    const int N = a.ring_size;
    int32_t head = a.ring_state[0] % N;
    if (head < 0) head += N;
    const int32_t count = min(max(a.ring_state[1], 0), N);

    int64_t sum = 0, total_rows, total;
    for (int b = lo; b < hi; ++b) sum += max(a.new_len[b], 0);
    const int64_t row0 = plan_scan(sum, scratch, &total_rows);
    int64_t row = row0, need = 0, freed = 0;
    for (int b = lo; b < hi; ++b) {
        const PlanSeq s = plan_load(a, b);
        row_start[b] = (int32_t)min(row, (int64_t)a.rows);
        row += s.n;
        const int f = s.n > 0 && row > a.rows ? PCG_FLAG_NO_ROWS : s.blocks > a.max_blocks ? PCG_FLAG_TOO_LONG : 0;
        flag[b] = (uint8_t)f;
        if (!s.done && !f) need += max(s.blocks - s.held, (int64_t)0);
        if (s.done) freed += s.held;
    }
    if (tid == 0) row_start[B] = (int32_t)min(total_rows, (int64_t)a.rows);
    int64_t total_freed;
    int64_t need_at = plan_scan(need, scratch, &total), freed_at = plan_scan(freed, scratch, &total_freed);
    int64_t granted = 0;
    for (int b = lo; b < hi; ++b) {
        const PlanSeq s = plan_load(a, b);
        if (s.done) {
            offset[b] = (int32_t)min(freed_at, (int64_t)N);
            freed_at += s.held;
        } else if (!flag[b]) {
            const int64_t want = max(s.blocks - s.held, (int64_t)0);
            offset[b] = (int32_t)min(need_at, (int64_t)N);
            need_at += want;
            if (want > 0 && need_at > count)
                flag[b] = PCG_FLAG_NO_BLOCKS;
            else
                granted += want;
        }
    }
    int64_t taken;
    plan_scan(granted, scratch, &taken);  // its barriers also publish the shared arrays
    if (blockIdx.x == 0 && tid == 0) {
        a.out_ring_state[0] = (int32_t)((head + taken) % N);
        a.out_ring_state[1] = (int32_t)(count - taken + min(total_freed, (int64_t)(N - count)));  // what was dropped is not free
        a.out_row_start[B] = row_start[B];
    }
    const int gtid = blockIdx.x * kPlanThreads + tid, gthreads = gridDim.x * kPlanThreads;
    for (int b = gtid; b < B; b += gthreads) {
        const PlanSeq s = plan_load(a, b);
        const int f = flag[b];
        a.out_cached_len[b] = (int32_t)min(s.base, (int64_t)0x7fffffff);
        a.out_kv_len[b] = s.done || f ? 0 : (int32_t)(s.base + s.n);
        a.out_held[b] = s.done ? 0 : f ? s.held : (int32_t)max(s.blocks, (int64_t)s.held);
        a.out_row_start[b] = row_start[b];
        if (a.out_flags) a.out_flags[b] = f;
    }
    const int lane = tid & 31;
    for (int b = gtid >> 5; b < B; b += gthreads >> 5) {  // one warp per sequence
        const PlanSeq s = plan_load(a, b);
        int32_t *entry = a.block_table + (int64_t)b * a.max_blocks;
        if (s.done) {  // never more than the ring has room for behind its free entries
            const int room = N - count - offset[b];
            for (int i = lane; i < min(s.held, room); i += 32) a.free_ring[((int64_t)head + count + offset[b] + i) % N] = entry[i];
        } else if (!flag[b]) {
            const int want = (int)max(s.blocks - s.held, (int64_t)0);
            for (int i = lane; i < want; i += 32) entry[s.held + i] = a.free_ring[((int64_t)head + offset[b] + i) % N];
        }
    }
    for (int64_t r = gtid; r < a.rows; r += gthreads) {
        int32_t slot = -1, pos = -1;
        if (r < row_start[B]) {
            int b = 0, end = B - 1;  // the last sequence that starts at or before r: empty ones share their start
            while (b < end) {
                const int mid = (b + end + 1) >> 1;
                if (row_start[mid] <= r)
                    b = mid;
                else
                    end = mid - 1;
            }
            if (!flag[b]) {
                const PlanSeq s = plan_load(a, b);
                const int64_t p = s.base + (r - row_start[b]);
                const int j = (int)(p / a.block_size);
                // blocks handed out by this call come from the ring: another block may not have written the entry yet
                const int32_t block = j < s.held ? a.block_table[(int64_t)b * a.max_blocks + j]
                                                 : a.free_ring[((int64_t)head + offset[b] + j - s.held) % N];
                pos = (int32_t)p;
                slot = block * a.block_size + (int)(p % a.block_size);
            }
        }
        a.out_slots[r] = slot;
        if (a.out_positions) a.out_positions[r] = pos;
    }
}

// ---------------------------------------------------------------------------------------------- append
// A copy: thread = one 16-byte vector of a token's keys and the same one of its values.  Consecutive threads walk a
// token's heads, so a warp reads 512 consecutive bytes of each input and writes whole rows of head_dim elements.
// What bounds it: HBM, rows * kv_heads * head_dim * 4 elements of traffic (33,001 rows of 8 x 128 bf16: 44.8 us, 6.03 TB/s,
// 94 % of the measured copy).
__global__ void __launch_bounds__(256) cache_append_kernel(const uint4 *k, int64_t k_stride, const uint4 *v, int64_t v_stride,
                                                           int32_t rows, const int32_t *slots, uint4 *kc, uint4 *vc,
                                                           int64_t n_slots, int bs_shift, int heads, int vecs) {
    const int per_row = heads * vecs;  // 16-byte vectors of a token
    const int64_t total = (int64_t)rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per_row;
        const int c = (int)(i - r * per_row), h = c / vecs, w = c - h * vecs;
        const int64_t slot = slots[r];
        if (slot < 0 || slot >= n_slots) continue;
        const int64_t block = slot >> bs_shift, at = slot & ((1 << bs_shift) - 1);
        const int64_t to = (((block * heads + h) << bs_shift) + at) * vecs + w;
        const uint4 x = k[r * k_stride + c], y = v[r * v_stride + c];
        kc[to] = x;
        vc[to] = y;
    }
}

// ---------------------------------------------------------------------------------------------- host
pcg_status check_here(const char *who, const void *p) {
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    cudaPointerAttributes at;
    e = cudaPointerGetAttributes(&at, p);
    if (e != cudaSuccess) return cuda_fail(e, "cudaPointerGetAttributes");
    if ((at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) || at.device != dev) {
        set_error("%s: the tensors must be memory of device %d, which is current", who, dev);
        return PCG_ERR_INVALID_ARG;
    }
    return PCG_OK;
}

bool valid_block_size(int32_t n) { return n >= 16 && n <= 256 && (n & (n - 1)) == 0; }

pcg_status check_cache(const char *who, const pcg_cache *c) {
    if (!c || !c->k || !c->v || ((uintptr_t)c->k & 15u) || ((uintptr_t)c->v & 15u)) {
        set_error("%s: the cache is null, or its arrays are null or not 16-byte aligned", who);
        return PCG_ERR_INVALID_ARG;
    }
    if (!valid_dtype(c->dtype) || !valid_block_size(c->block_size) || c->n_blocks < 1 || c->kv_heads < 1 ||
        c->kv_heads > 1024 || c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 ||
        (int64_t)c->n_blocks * c->block_size > 0x7fffffff) {
        set_error("%s: bad cache (dtype %d, %d blocks of %d tokens, %d heads of %d): block_size is 16, 32, 64, 128 or "
                  "256, head_dim a multiple of 8 up to 256, kv_heads 1 to 1024, and the slots fit 31 bits",
                  who, (int)c->dtype, c->n_blocks, c->block_size, c->kv_heads, c->head_dim);
        return PCG_ERR_INVALID_ARG;
    }
    return PCG_OK;
}

pcg_status check_rows(const char *who, const char *name, const void *p, int64_t stride, int32_t heads, int32_t d,
                      pcg_dtype dtype) {
    const int64_t esz = (int64_t)dtype_bytes(dtype);
    if (!p || ((uintptr_t)p & 15u) || stride < (int64_t)heads * d || stride > ((int64_t)1 << 36) || (stride * esz) % 16) {
        set_error("%s: %s is null, not 16-byte aligned, or its stride of %lld elements is under heads * head_dim or not "
                  "a multiple of 16 bytes", who, name, (long long)stride);
        return PCG_ERR_INVALID_ARG;
    }
    return PCG_OK;
}

}  // namespace pcg

using namespace pcg;

extern "C" pcg_status pcg_cache_plan(int32_t B, const int32_t *cached_len, const int32_t *accept_len, const int32_t *new_len,
                                     const int32_t *held, int32_t block_size, int32_t max_blocks, int32_t *block_table,
                                     int32_t *free_ring, int32_t ring_size, const int32_t *ring_state, int32_t rows,
                                     int32_t *out_cached_len, int32_t *out_kv_len, int32_t *out_held,
                                     int32_t *out_row_start, int32_t *out_slots, int32_t *out_positions,
                                     int32_t *out_ring_state, int32_t *out_flags, pcg_stream stream) {
    if (B < 0 || rows < 0 || ring_size < 1 || max_blocks < 1 || !valid_block_size(block_size) ||
        (int64_t)max_blocks * block_size > 0x7fffffff) {
        set_error("pcg_cache_plan: need B, rows >= 0, ring_size, max_blocks >= 1, block_size 16, 32, 64, 128 or 256 and "
                  "max_blocks * block_size < 2^31 (B=%d rows=%d ring_size=%d max_blocks=%d block_size=%d)",
                  B, rows, ring_size, max_blocks, block_size);
        return PCG_ERR_INVALID_ARG;
    }
    if (!free_ring || !ring_state || !out_row_start || !out_ring_state || (rows > 0 && !out_slots) ||
        (B > 0 && (!cached_len || !new_len || !held || !block_table || !out_cached_len || !out_kv_len || !out_held))) {
        set_error("pcg_cache_plan: null pointer");
        return PCG_ERR_INVALID_ARG;
    }
    if (out_cached_len == cached_len || out_held == held || out_ring_state == ring_state || out_kv_len == cached_len ||
        out_kv_len == new_len || out_kv_len == held || out_cached_len == new_len) {
        if (B > 0) {
            set_error("pcg_cache_plan: outputs may not overlap inputs");
            return PCG_ERR_INVALID_ARG;
        }
    }
    if (B > kPlanMaxB) {
        set_error("pcg_cache_plan: B=%d exceeds the supported %d sequences", B, kPlanMaxB);
        return PCG_ERR_UNSUPPORTED;
    }
    pcg_status st = check_here("pcg_cache_plan", out_ring_state);
    if (st != PCG_OK) return st;
    const PlanArgs a{B, block_size, max_blocks, ring_size, rows, cached_len, accept_len, new_len, held, ring_state,
                     block_table, free_ring, out_cached_len, out_kv_len, out_held, out_row_start, out_slots,
                     out_positions, out_ring_state, out_flags};
    const size_t smem = (size_t)(2 * B + 1) * 4 + B;
    cudaError_t e = cudaSuccess;
    if (smem > 48 * 1024)
        e = cudaFuncSetAttribute(cache_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (2 * kPlanMaxB + 1) * 4 + kPlanMaxB);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute (cache plan)");
    const int64_t work = (int64_t)rows + (int64_t)B * 8;
    const int grid = (int)(work < 2 * kPlanThreads ? 1 : work / (2 * kPlanThreads) < 148 ? work / (2 * kPlanThreads) : 148);
    cache_plan_kernel<<<grid, kPlanThreads, smem, (cudaStream_t)stream>>>(a);
    e = cudaGetLastError();
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, "launching the cache plan kernel");
}

extern "C" pcg_status pcg_cache_append(const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t rows,
                                       const int32_t *slots, const pcg_cache *cache, pcg_stream stream) {
    pcg_status st = check_cache("pcg_cache_append", cache);
    if (st != PCG_OK) return st;
    if (rows < 0 || (rows > 0 && !slots)) {
        set_error("pcg_cache_append: rows < 0, or null slots");
        return PCG_ERR_INVALID_ARG;
    }
    if (rows == 0) return PCG_OK;
    st = check_rows("pcg_cache_append", "k", k, k_stride, cache->kv_heads, cache->head_dim, cache->dtype);
    if (st == PCG_OK) st = check_rows("pcg_cache_append", "v", v, v_stride, cache->kv_heads, cache->head_dim, cache->dtype);
    if (st == PCG_OK) st = check_here("pcg_cache_append", cache->k);
    if (st != PCG_OK) return st;
    const int64_t esz = (int64_t)dtype_bytes(cache->dtype);
    const int vecs = (int)(cache->head_dim * esz / 16);
    const int64_t total = (int64_t)rows * cache->kv_heads * vecs, blocks = (total + 255) / 256;
    const int grid = (int)(blocks < 148 * 8 * 8 ? blocks : 148 * 8 * 8);
    cache_append_kernel<<<grid, 256, 0, (cudaStream_t)stream>>>(
        (const uint4 *)k, k_stride * esz / 16, (const uint4 *)v, v_stride * esz / 16, rows, slots, (uint4 *)cache->k,
        (uint4 *)cache->v, (int64_t)cache->n_blocks * cache->block_size, __builtin_ctz(cache->block_size), cache->kv_heads, vecs);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, "launching the cache append kernel");
}
