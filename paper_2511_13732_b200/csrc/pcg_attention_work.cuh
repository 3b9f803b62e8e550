// How the attention kernels share their work out and join what they shared: items, the cut of a call's work into one equal
// run per block, a block's walk through its run, the workspace, and the kernel that joins the parts of an item.
#pragma once

#include <cuda_bf16.h>

#include "pcg_attention.cuh"

namespace pcg {

constexpr int kTile = 128;       // rows of a row tile = lanes of tensor memory; keys of a key tile of an item with two
constexpr int kHalf = 64;        // keys of a key tile of an item with one row tile; rows of one copy at the most
constexpr int kMaxBlocks = 148;  // blocks of the main kernel: one per SM of a B200 (more or fewer SMs only change the pace)

// ---------------------------------------------------------------------------------------------- workspace
struct Run {        // one block's key tiles
    int64_t first;  // number of its first 64 keys among those of the call
    int32_t b, h, pair, tile;  // where that is (tile: in 64 keys)
};
struct WorkspaceHead {
    Run run[kMaxBlocks + 1];     // the last begins behind the last keys
    int32_t failed[kMaxBlocks];  // set where a bounded wait ran out: the call's outputs are then NaN
};
// Partial sums: [block][2: a part that does not begin its item, one that does][2 * 128 rows], D sums each stored
// [D][256] so that a warp's 32 rows are adjacent, then reference and sum of weights.
constexpr int kPartRows = 2 * kTile;
template <int D>
__host__ __device__ constexpr size_t part_floats() {
    return (size_t)kPartRows * (D + 2);
}
constexpr size_t kHeadBytes = (sizeof(WorkspaceHead) + 255) / 256 * 256;

__device__ __forceinline__ float *part_base(void *ws, int block, int which, int D) {
    return reinterpret_cast<float *>((char *)ws + kHeadBytes) + ((size_t)block * 2 + which) * kPartRows * (D + 2);
}

// ---------------------------------------------------------------------------------------------- items
__host__ __device__ __forceinline__ int pairs_of(int n, int TQ) { return (n + 2 * TQ - 1) / (2 * TQ); }
// Keys of pair p in units of 64: up to what its last row sees, in whole key tiles, and one of them where it sees nothing.
__device__ __forceinline__ int tiles_of(int n, int len, int TQ, int p) {
    const int tokens = min(n - p * 2 * TQ, 2 * TQ), lim = len - n + p * 2 * TQ + tokens;
    if (tokens > TQ) return lim <= kTile ? 2 : (lim + kTile - 1) / kTile * 2;
    return lim <= kHalf ? 1 : (lim + kHalf - 1) / kHalf;
}

// Sum over 0 <= i < n of floor((a i + b) / 128), a, b >= 0.  a a power of two, as it is where the query heads a key head
// are: floor((i + floor(b / a)) / (128 / a)), in closed form.  Else the sum of floors of a line by the Euclidean algorithm
// (points below the line are points beside it with the axes exchanged, and a and the divisor shrink as in a greatest common
// divisor), its first step by shifts; what is left fits 32 bits.
__device__ __forceinline__ int64_t floor_sum_128(uint32_t n, uint32_t a, int64_t b) {
    const int64_t nn = n;
    if ((a & (a - 1)) == 0) {
        if (a >= 128) return nn * (nn - 1) / 2 * (a >> 7) + nn * (b >> 7);
        const int k = 7 - (31 - __clz(a));  // 128 / a = 2^k
        auto upto = [&](int64_t x) {  // sum over 0 <= j < x of floor(j / 2^k)
            const int64_t q = x >> k, r = x & ((1 << k) - 1);
            return ((q * (q - 1) / 2) << k) + r * q;
        };
        const int64_t c = b >> (7 - k);
        return upto(nn + c) - upto(c);
    }
    int64_t s = nn * (nn - 1) / 2 * (a >> 7) + nn * (b >> 7);
    a &= 127;
    int64_t y = (int64_t)a * n + (b & 127);
    uint32_t m = a, x = 128;  // from here: sum over 0 <= i < y / 128 of floor((128 i + y % 128) / a), and so on
    uint32_t c = (uint32_t)(y & 127);
    n = (uint32_t)(y >> 7);
    while (n > 0) {
        const int64_t k = n;
        s += k * (k - 1) / 2 * (x / m) + k * (c / m);
        x %= m;
        c %= m;
        const uint64_t z = (uint64_t)x * n + c;
        if (z < m) break;
        n = (uint32_t)(z / m);
        c = (uint32_t)(z % m);
        const uint32_t t = x;
        x = m;
        m = t;
    }
    return s;
}
// The same of a sequence's first p pairs together.
inline __device__ int64_t tiles_before(int n, int len, int TQ, int p) {
    const int step = 2 * TQ, whole = n / step, q = min(p, whole);  // `whole` pairs of 2 * TQ tokens, then one of fewer
    // pairs whose last row sees at most one tile of keys count 1 each: (i + 1) * step <= 128 - (len - n)
    const int base = len - n;
    const int head = base >= kTile ? 0 : (int)min((int64_t)q, (kTile - (int64_t)base) / step);
    int64_t s = head;
    if (q > head) s += floor_sum_128(q - head, step, base + (int64_t)(head + 1) * step + kTile - 1);
    s *= 2;
    if (p > whole) s += tiles_of(n, len, TQ, whole);
    return s;
}

// ---------------------------------------------------------------------------------------------- the cut
// What an item costs beside its keys (fetching queries, the first and the last tile's latency, writing out), in units of 64
// keys: measured at 6,500 to 7,800 cycles for 3,500 a key tile of 128.  Blocks get at least kLeast units: fewer, and a
// short call's parts cost more to join than they save.
constexpr int kItemUnits = 4, kLeast = 4;

// By all threads of the block: where runs `block` and `block + 1` begin, to out[0] and out[1].  `scratch` holds B
// int64_t and B int32_t (192 KB of shared memory at the most).
inline __device__ void cut_work(const AttnArgs &a, int TQ, int64_t *scratch, int64_t *warp_units, int64_t *warp_items, Run *out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, B = a.B;
    int64_t *units = scratch;                                 // [B] of the sequences before b
    int32_t *items = reinterpret_cast<int32_t *>(units + B);  // [B] items of one head of the sequences before b
    const int per = (B + threads - 1) / threads, lo = min(B, tid * per), hi = min(B, lo + per);
    int64_t usum = 0, isum = 0;
    for (int b = lo; b < hi; ++b) {
        units[b] = usum;
        items[b] = (int32_t)isum;
        int begin, n, len;
        attn_sequence(a, b, begin, n, len);
        const int pairs = pairs_of(n, TQ);
        if (n > 0) {
            const int64_t tiles = pairs == 1 ? tiles_of(n, len, TQ, 0) : tiles_before(n, len, TQ, pairs);
            usum += (tiles + (int64_t)kItemUnits * pairs) * a.kv_heads;
            isum += pairs;
        }
    }
    int64_t uinc = usum, iinc = isum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, uinc, o), i = __shfl_up_sync(0xffffffffu, iinc, o);
        if (lane >= o) {
            uinc += u;
            iinc += i;
        }
    }
    if (lane == 31) {
        warp_units[warp] = uinc;
        warp_items[warp] = iinc;
    }
    __syncthreads();
    int64_t ubase = uinc - usum, ibase = iinc - isum, total = 0, all_items = 0;
    for (int w = 0; w < threads / 32; ++w) {
        if (w < warp) {
            ubase += warp_units[w];
            ibase += warp_items[w];
        }
        total += warp_units[w];
        all_items += warp_items[w];
    }
    for (int b = lo; b < hi; ++b) {
        units[b] += ubase;
        items[b] += (int32_t)ibase;
    }
    __syncthreads();
    if (warp < 2) {  // a warp for each of the two
        const int blocks = (int)max((int64_t)1, min((int64_t)kMaxBlocks, total / kLeast)), c = blockIdx.x + warp;
        Run r{total - (int64_t)kItemUnits * a.kv_heads * all_items, 0, 0, 0, 0};  // behind the last keys
        // (64-bit divisions are calls; below 2^31 units, 32 bits do)
        const bool small = total <= 0x7fffffff;
        const int64_t each = small ? (int64_t)((uint32_t)total / (uint32_t)blocks) : total / blocks;
        const uint32_t left = (uint32_t)(total - each * blocks);
        const int64_t u = c >= blocks ? total : each * c + left * (uint32_t)c / (uint32_t)blocks;
        if (u < total) {
            int x = 0, y = B - 1;  // the last sequence whose units begin at or before u: empty ones share their number
            while (x < y) {
                const int mid = (x + y + 1) >> 1;
                if (units[mid] <= u)
                    x = mid;
                else
                    y = mid - 1;
            }
            int begin, n, len;
            attn_sequence(a, x, begin, n, len);
            const int pairs = pairs_of(n, TQ);
            const int64_t tiles = pairs == 1 ? tiles_of(n, len, TQ, 0) : tiles_before(n, len, TQ, pairs);
            const int64_t per_head = tiles + (int64_t)kItemUnits * pairs, in = u - units[x];
            const int h = small ? (int)((uint32_t)in / (uint32_t)per_head) : (int)(in / per_head);
            const int64_t rest = in - h * per_head;
            // the pair: of [p, p + count) in steps of a 32nd, by the lanes
            int p = 0, count = pairs;
            int64_t head_tiles = 0;
            while (count > 1) {
                const int step = (count + 31) / 32, mine = p + lane * step;
                const int64_t before = lane * step < count && mine > 0 ? tiles_before(n, len, TQ, mine) : 0;
                const bool below = lane * step < count && before + (int64_t)kItemUnits * mine <= rest;
                const int top = 31 - __clz(__ballot_sync(0xffffffffu, below));  // lane 0's always is
                head_tiles = __shfl_sync(0xffffffffu, before, top);
                count = min(step, count - top * step);
                p += top * step;
            }
            // an item's own units come first: a cut within them leaves the whole item to the run behind it
            int64_t tile = max((int64_t)0, rest - head_tiles - (int64_t)kItemUnits * p - kItemUnits);
            if (n - p * 2 * TQ > TQ) tile &= ~(int64_t)1;  // a whole key tile
            r.first = units[x] - (int64_t)kItemUnits * a.kv_heads * items[x] + h * tiles + head_tiles + tile;
            r.b = x;
            r.h = h;
            r.pair = p;
            r.tile = (int)tile;
        }
        if (lane == 0) out[warp] = r;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // copies land in the scratch's place
    __syncthreads();
}

// A block's run of units, item by item: the same walk in every role.
struct Segment {
    int b, h, pair, begin, n, len;
    int t0, nt;   // the first key tile of this part, how many
    bool whole;   // the part is the item
    bool two;     // two row tiles, key tiles of 128 keys; else of 64
};
struct Walk {
    int b, h, pair, tile, left;
    int begin, n, len;
    __device__ __forceinline__ void start(const AttnArgs &a, const Run &r, const Run &next) {
        b = r.b;
        h = r.h;
        pair = r.pair;
        tile = r.tile;
        left = (int)min(next.first - r.first, (int64_t)0x7fffffff);
        if (left > 0) attn_sequence(a, b, begin, n, len);
    }
    __device__ __forceinline__ bool next(const AttnArgs &a, int TQ, Segment &s) {
        if (left <= 0) return false;
        s.b = b;
        s.h = h;
        s.pair = pair;
        s.begin = begin;
        s.n = n;
        s.len = len;
        s.two = n - pair * 2 * TQ > TQ;
        const int all = tiles_of(n, len, TQ, pair), nt = min(left, all - tile);
        s.whole = nt == all;
        s.t0 = s.two ? tile >> 1 : tile;
        s.nt = s.two ? max(nt >> 1, 1) : nt;
        left -= nt;
        tile = 0;
        if (left > 0 && ++pair == pairs_of(n, TQ)) {
            pair = 0;
            if (++h == a.kv_heads) {
                h = 0;
                do {
                    if (++b >= a.B) {  // row starts that overlap may have been counted for more than there is
                        left = 0;
                        break;
                    }
                    attn_sequence(a, b, begin, n, len);
                } while (n == 0);
            }
        }
        return true;
    }
};

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (BF16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ---------------------------------------------------------------------------------------------- combine
// N values, rounded once.
template <int N>
__device__ __forceinline__ void store_values(float *p, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<float2 *>(p + i) = make_float2(x[i], x[i + 1]);
}
template <int N>
__device__ __forceinline__ void store_values(uint16_t *p, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<uint32_t *>(p + i) = pack2<true>(x[i], x[i + 1]);
}
template <int N>
__device__ __forceinline__ void store_values(f16_t *p, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<uint32_t *>(p + i) = pack2<false>(x[i], x[i + 1]);
}

// Block (c, y, z): the item that block c of the main kernel began and did not end, if there is one; a quarter of the head
// dimensions (y), every other 32 rows (z); thread = row (lane) and D / 32 dimensions (warp).  What bounds it is the latency
// of the parts' loads, which do not depend on each other.
constexpr int kCombineThreads = 256, kCombineDims = 4, kCombineRows = 2;

template <int D, typename T>
__global__ void __launch_bounds__(kCombineThreads) attention_combine_kernel(const __grid_constant__ AttnArgs a, void *ws) {
    constexpr int N = D / (8 * kCombineDims);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const WorkspaceHead *head = reinterpret_cast<const WorkspaceHead *>(ws);
    const int tid = threadIdx.x, lane = tid & 31, dims = (blockIdx.y * 8 + (tid >> 5)) * N;
    const int c = blockIdx.x;
    const Run next = head->run[c + 1];
    const int64_t begun = head->run[c].first, all = head->run[kMaxBlocks].first;
    if (__syncthreads_or(tid < kMaxBlocks && head->failed[tid])) {  // no row may pass for a result
        const uint32_t nan2 = 0x7fff7fffu;  // NaN in all three types
        const int64_t vecs = (int64_t)a.rows * a.q_heads * (D * (int)sizeof(T) / 16), blocks = (int64_t)gridDim.x * gridDim.y * gridDim.z;
        for (int64_t i = (((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + c) * kCombineThreads + tid; i < vecs;
             i += blocks * kCombineThreads)
            reinterpret_cast<uint4 *>(a.out)[i] = make_uint4(nan2, nan2, nan2, nan2);
        return;
    }
    if (next.first >= all || next.tile == 0 || next.first - next.tile < begun) return;
    const int G = a.q_heads / a.kv_heads, TQ = kTile / G;
    int begin, n, len;
    attn_sequence(a, next.b, begin, n, len);
    const int64_t end = next.first - next.tile + tiles_of(n, len, TQ, next.pair);
    int last = c + 1;  // the block that ends the item
    while (last + 1 < kMaxBlocks && head->run[last + 1].first < end) ++last;
    const int tokens = min(n - next.pair * 2 * TQ, 2 * TQ);
    const int rows = tokens > TQ ? kPartRows : kTile;
    // the first part lies among its block's parts that begin an item, the others among those that do not
    const float *first = part_base(ws, c, 1, D), *rest = part_base(ws, c + 1, 0, D);
    constexpr int64_t kStride = 2 * (int64_t)part_floats<D>();
    const int more = last - c;
    for (int r0 = blockIdx.z * 32; r0 < rows; r0 += 32 * kCombineRows) {
        const int r = r0 + lane, in = r & (kTile - 1);
        const int tok = (r / kTile) * TQ + in / G;
        if (in / G >= TQ || tok >= tokens) continue;
        constexpr int64_t kM = (int64_t)D * kPartRows, kL = kM + kPartRows;
        const float m0 = first[kM + r];
        float m = m0;
#pragma unroll 8
        for (int k = 0; k < more; ++k) m = fmaxf(m, rest[k * kStride + kM + r]);
        float f = m0 == kNegInf ? 0.f : m0 == m ? 1.f : ex2(m0 - m);
        float l = first[kL + r] * f, o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = first[(dims + i) * kPartRows + r] * f;
#pragma unroll 4
        for (int k = 0; k < more; ++k) {
            const float *p = rest + k * kStride;
            const float mk = p[kM + r];
            f = mk == kNegInf ? 0.f : mk == m ? 1.f : ex2(mk - m);
            l += p[kL + r] * f;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] += p[(dims + i) * kPartRows + r] * f;
        }
        const int t_row = next.pair * 2 * TQ + tok;
        const bool empty = len - n + t_row + 1 <= 0;
        const float inv = 1.f / l;  // 0 / 0 where every score was -inf
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = empty ? 0.f : o[i] * inv;
        store_values((T *)a.out + (((int64_t)begin + t_row) * a.q_heads + next.h * G + in % G) * D + dims, o);
    }
}

// Launches behind the stream's last kernel without waiting for its end (the kernels wait for it themselves).
template <typename... KArgs, typename... Args>
cudaError_t launch_behind(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}


}  // namespace pcg
