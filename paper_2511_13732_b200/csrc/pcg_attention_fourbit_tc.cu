// Attention over the cache that holds 4.5 bits a value, on the 5th-generation tensor cores: bfloat16 and float16 queries, head
// dimensions 64 and 128, up to 48 query heads a key head.
//
// The products are turned round: keys, not rows, lie on the lanes of tensor memory.
//     S^T[key][row] = K[key][dim] Q^T[dim][row]        A = keys, one a lane, straight out of tensor memory
//     O^T[dim][row] += V^T[dim][key] P^T[key][row]     A = values, one dimension a lane, out of tensor memory
// So codes become operands without passing through shared memory a second time: a thread widens the codes of its own key (or
// value dimension), 2 values an instruction, multiplies them by their scales -- a code times a scale has six significant
// bits, exact in float16 -- and stores them to its own lane.  And a product is as wide as there are rows (16 to 48 columns),
// where rows on lanes would be padded to 128: four query heads of one token cost a quarter of 16 columns.
// The rows (queries, weights) are the small operand and come from shared memory.
//
// Work is shared out as in the 16-bit kernel: items of (sequence, key head, up to two SLOTS of 48 rows), every block an equal
// run of them, parts joined by a second kernel.  With rows for two slots both take every key tile of 128; with fewer, the
// slots take the key tiles in turn and their sums meet at the end.
//
// Warps 0-7    softmax, four a slot; a thread has one key of a tile and all the slot's rows.  A row's reference may lag its
//              maximum by 2^8, so a tile only needs the one bit "some score is further above": maxima are formed for an item's
//              first tile and where that bit is set.
// Warps 8-11   keys, 12-15 values: codes to operands.
// Warp 16      copies: pages of 16 tokens are contiguous, whatever the block size; a tile is 8 of them.
// Warp 17      products for the scores, 19 for the outputs.  (By one warp, each product also waited for the other kind's turn.)
// Warp 18      queries: rounded to float16 with a power of two for each row.
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "pcg_attention_work.cuh"
#include "pcg_fourbit.cuh"
#include "pcg_tcgen05.cuh"

namespace pcg {

namespace {

constexpr int kCols = kFourbitCols, kKeys = 128;  // rows of a slot; keys of a tile
constexpr int kFourbitThreads = 32 * 20;
// Registers: 640 threads are launched with 96; the softmax's 8 warps take 144, which the other 12 leave by keeping 64
// (8 * 32 * 144 + 12 * 32 * 64 = 640 * 96).
#define PCG_SOFTMAX_REGISTERS "144"
#define PCG_OTHER_REGISTERS "64"
constexpr int kScoreBufs = 3;  // scores in tensor memory: those of the tiles and slots in turn
constexpr int kPBytes = kKeys * 128;  // weights of a tile: 64 columns of 16 bits a key, 128-byte swizzled
constexpr float kSlack = 8.f;         // the reference may lag the maximum by a factor 2^8 before sums are scaled
// Weights are kept 2^7 higher than the reference says, out of the range where float16 loses bits: 2^8 above the reference is
// then 2^15 at most.  The sums carry the same factor, so it cancels.
constexpr float kLift = 7.f;
constexpr int kFourItemUnits = 8, kFourLeast = 8;

template <int D>
struct Sizes4 {
    static constexpr int kQSlot = D / 64 * kCols * 128;  // queries of a slot: D / 64 parts of 48 rows x 128 bytes
    static constexpr int kQBytes = 4 * kQSlot;           // two slots, of this item and the next
    static constexpr int kWeights = 4 * kPBytes;         // two slots, two tiles each
    static constexpr int kStage = 8 * page_bytes(D);
    static constexpr int kScales = D / 16 * kKeys * 2;   // of a tile's values, as float16
    static constexpr int kStages = D == 128 ? 5 : 12;
    static constexpr int kSmem = kQBytes + kWeights + 2 * kScales + kStages * kStage;
    static_assert(kSmem >= kAttnMaxB * 12, "the cut's scratch");
};

// An item's rows: tokens in all, and those of slot 0.
struct Split {
    int tokens, tq;
    bool two;
};
__device__ __forceinline__ Split split_of(int n, int pair, int TQ) {
    Split s;
    s.tokens = min(n - pair * 2 * TQ, 2 * TQ);
    s.two = s.tokens > TQ;
    s.tq = s.two ? (s.tokens + 1) / 2 : s.tokens;
    return s;
}

// Parts of items: [block][2: one that does not begin its item, one that does][2 * 48 rows][D] sums, then references, then sums
// of weights.
constexpr int kFourPartRows = 2 * kCols;
template <int D>
__device__ __forceinline__ float *four_part(void *ws, int block, int which) {
    return reinterpret_cast<float *>((char *)ws + kHeadBytes) + ((size_t)block * 2 + which) * kFourPartRows * (D + 2);
}

// bar_wait_hot with a poll that may sleep for 10 us: of 20 warps most wait, and their polls would take the issue slots (and
// instruction cache) of those that work.
constexpr uint32_t kPollTime = 10000;
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int *failed) {
#pragma unroll 1
    for (uint32_t i = 0; i < (1u << 17); ++i) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity), "r"(kPollTime)
            : "memory");
        if (done) return true;
        if (*failed) return false;
    }
    *failed = 1;
    return false;
}
__device__ __forceinline__ void warps_meet(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// Whether any of a slot's 128 threads says so.
__device__ __forceinline__ bool slot_any(int id, bool mine) {
    int r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((int)mine), "r"(id)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ float warp_max(float x) {  // NaN only where all are
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    const __half2 r = __hmul2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// Sums of N (8 or 16) columns, held in pairs, over a warp's lanes: lane i < N ends with column i's.
template <int N>
__device__ __forceinline__ float column_sums(const uint64_t *x, int lane) {
    float v[N];
#pragma unroll
    for (int i = 0; i < N; i += 2) unpair(x[i / 2], v[i], v[i + 1]);
#pragma unroll
    for (int w = N / 2; w >= 1; w >>= 1) {
        const bool up = lane & w;
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const float give = up ? v[i] : v[i + w], keep = up ? v[i + w] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, w);
        }
    }
#pragma unroll
    for (int w = N; w < 32; w <<= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], w);
    return v[0];
}
__device__ __forceinline__ void tmem_ld8(uint32_t addr, uint32_t *v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : PCG_R8(v, 0) : "r"(addr));
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t *v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), PCG_W8(v, 0) : "memory");
}
// N (8, 16, 32 or 48) columns of the warp's lanes, waited for.
template <int N>
__device__ __forceinline__ void load_columns(uint32_t addr, uint32_t (&v)[N]) {
    if (N == 8) tmem_ld8(addr, v);
    if (N >= 32) tmem_ld32(addr, v);
    if (N == 16 || N == 48) tmem_ld16(addr + (N & 32), v + (N & 32));
    tmem_wait_ld();
    tmem_loaded<N>(v);
}

template <typename T>
__device__ __forceinline__ T round_to(float x);
template <>
__device__ __forceinline__ uint16_t round_to<uint16_t>(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
template <>
__device__ __forceinline__ f16_t round_to<f16_t>(float x) { return f16_t{__half_as_ushort(__float2half_rn(x))}; }

template <int D, typename T>
__global__ void __launch_bounds__(kFourbitThreads, 1)
    attention_fourbit_kernel(const __grid_constant__ AttnArgs a, float v_scale, void *ws) {
    using Z = Sizes4<D>;
    constexpr int S = Z::kStages, kPage = page_bytes(D), kValueWarps = D / 32;
    // instruction descriptors: D = fp32, A and B float16, M = 128; B K-major (queries), MN-major (weights); N is added
    constexpr uint32_t kIdescQK = (1u << 4) | ((kKeys >> 4) << 24), kIdescPV = kIdescQK | (1u << 16);

    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ int64_t warp_units[kFourbitThreads / 32], warp_items[kFourbitThreads / 32];
    __shared__ Run run[2];
    __shared__ __align__(8) uint64_t bars[2 * S + 32];
    __shared__ float q_by[2][2][kCols];      // of an item's rows (buffer, slot): what a product is multiplied by, 0 for padding
    __shared__ int q_lim[2][2][kCols];       // ... how many keys it sees
    __shared__ float4 col[2][kCols / 2];     // of a slot's column pairs: factors, then -reference + lift; later the joined factors
    __shared__ float col_m[2][2][kCols], col_l[2][2][kCols], col_f[2][kCols];  // (part's parity, slot): references, sums
    __shared__ float warp_col[2][4][kCols];
    __shared__ uint32_t tmem_slot;
    __shared__ int failed_flag;
    volatile int *failed = &failed_flag;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t qbuf = smem_u32(smem_raw), pbuf = qbuf + Z::kQBytes, scale_buf = pbuf + Z::kWeights, ring = scale_buf + 2 * Z::kScales, bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };         // a stage has landed
    auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };  // ... been read
    const uint32_t more = bar0 + 16u * S;
    auto k_full = [&](int i) { return more + 8u * i; };           // operands of a tile's keys are in place (two buffers)
    auto k_empty = [&](int i) { return more + 16u + 8u * i; };
    auto v_full = [&](int i) { return more + 32u + 8u * i; };
    auto v_empty = [&](int i) { return more + 48u + 8u * i; };
    auto s_full = [&](int i) { return more + 64u + 8u * i; };     // scores are complete (a ring of three)
    auto s_empty = [&](int i) { return more + 88u + 8u * i; };    // ... read
    auto p_full = [&](int s, int i) { return more + 112u + 16u * s + 8u * i; };  // a slot's weights are in place (two buffers)
    auto p_empty = [&](int s, int i) { return more + 144u + 16u * s + 8u * i; };
    auto o_full = [&](int s) { return more + 176u + 8u * s; };    // a slot's last product of a part is complete
    auto o_empty = [&](int s) { return more + 192u + 8u * s; };   // its outputs have been read
    auto q_full = [&](int i) { return more + 208u + 8u * i; };    // an item's queries are in place (two buffers)
    auto q_empty = [&](int i) { return more + 224u + 8u * i; };
    const uint32_t drain = more + 240u;  // of the two warps that issue products

    if (tid == 0) {
        for (int i = 0; i < 2 * S + 32; ++i) {
            const uint32_t bar = bar0 + 8u * i;
            uint32_t count = 1;  // by the hardware, or one thread
            if (bar >= empty_bar(0) && bar < more) count = 4 + kValueWarps;
            if (bar == k_full(0) || bar == k_full(1)) count = 4;
            if (bar == v_full(0) || bar == v_full(1)) count = kValueWarps;
            if (bar >= s_empty(0) && bar <= p_full(1, 1)) count = 4;
            if (bar == o_empty(0) || bar == o_empty(1)) count = 4;
            if (bar == q_empty(0) || bar == q_empty(1)) count = 9;
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed_flag = (qbuf & 1023u) != 0;  // never: the array is declared so
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_slot;
    auto k_col = [&](int i) { return tmem + (uint32_t)(i * 64); };
    auto v_col = [&](int i) { return tmem + (uint32_t)(128 + i * 64); };
    auto s_col = [&](int i) { return tmem + (uint32_t)(256 + i * kCols); };
    auto o_col = [&](int s) { return tmem + (uint32_t)(256 + (kScoreBufs + s) * kCols); };
    static_assert(256 + (kScoreBufs + 2) * kCols <= 512, "tensor memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int G = a.q_heads / a.kv_heads, TQ = kCols / G;
    cut_work<kFourItemUnits, kFourLeast>(a, TQ, reinterpret_cast<int64_t *>(smem_raw), warp_units, warp_items, run);
    if (tid == 0) reinterpret_cast<WorkspaceHead *>(ws)->run[blockIdx.x] = run[0];
    if (tid == 0 && blockIdx.x == kMaxBlocks - 1) reinterpret_cast<WorkspaceHead *>(ws)->run[kMaxBlocks] = run[1];
    Walk walk;
    walk.start(a, run[0], run[1]);
    Segment g;
    // the keys of a part: from the first tile's first on, up to (not with) the last
    auto first_key = [&](const Segment &g) { return g.t0 * (g.two ? 128 : 64); };
    auto last_key = [&](const Segment &g) { return g.two ? g.len : min(g.len, (g.t0 + g.nt) * 64); };
    auto tiles = [&](const Segment &g) { return g.two ? g.nt : (g.nt + 1) >> 1; };

    if (warp < 8) {
        // ------------------------------------------------------------------ softmax: thread = key of a tile
        asm volatile("setmaxnreg.inc.sync.aligned.u32 " PCG_SOFTMAX_REGISTERS ";");
        const int slot = warp >> 2, row = (warp & 3) * 32 + lane, wg_id = 1 + slot, wt = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t oc = o_col(slot) + lanes;
        uint32_t count = 0, outs = 0, outs_other = 0, part = 0;  // tiles of this slot, its outputs, the other's, parts so far
        uint32_t sb = 0, s_phase = 0;                             // buffer of the next scores (of either slot), its phase
        // After a wait that ran out the waits return at once; the role goes on to its end, since its warps meet at barriers.
        for (; walk.next(a, TQ, g); ++part) {
            const int qb = part & 1;
            const Split sp = split_of(g.n, g.pair, TQ);
            const int tokens = !g.two ? sp.tokens : slot ? sp.tokens - sp.tq : sp.tq, t_first = g.pair * 2 * TQ + (g.two && slot ? sp.tq : 0);
            const int rows = tokens * G;
            const int nt = tiles(g), first = g.two ? 0 : slot, step = g.two ? 1 : 2, k_first = first_key(g), k_end = last_key(g);
            const int qs = g.two ? slot : 0;  // whose queries
            const int least = min(g.len - g.n + t_first + 1, k_end);  // keys that every row sees
            const bool mine = first < nt, shared = !g.two && nt > 1;
            wait_for(q_full(qb), (part >> 1) & 1, failed);
            if (wt < kCols) {
                float *c = reinterpret_cast<float *>(&col[slot][wt >> 1]) + (wt & 1);
                c[0] = q_by[qb][qs][wt];
                c[2] = wt < rows ? kLift : kNegInf;  // padding weighs nothing
                col_m[qb][slot][wt] = kNegInf;
            }
            warps_meet(wg_id, 128);
            auto next_scores = [&]() {
                if (++sb == kScoreBufs) {
                    sb = 0;
                    s_phase ^= 1;
                }
            };
            if (slot) next_scores();  // slot 0's first tile's come before this one's
            // The part's tiles with N columns: as many as the slot has rows, or the next of 8, 16, 32, 48.  Their sums stay in
            // registers, and the scores of a tile.
            auto part_of = [&](auto columns) {
                constexpr int N = decltype(columns)::value;
                uint64_t l[N / 2];
#pragma unroll
                for (int i = 0; i < N / 2; ++i) l[i] = 0;
#pragma unroll 1
                for (int t = first; t < nt; t += step, ++count) {
                    wait_for(s_full(sb), s_phase, failed);
                    fence_after();
                    const int k0 = k_first + t * kKeys, key = k0 + row;
                    const uint32_t sc = s_col(sb) + lanes;
                    uint32_t x[N];
                    auto load = [&]() {
                        load_columns<N>(sc, x);
                        if (__builtin_expect(k0 + kKeys > least, 0)) {  // keys that a row does not see
#pragma unroll
                            for (int i = 0; i < N; ++i)
                                if (key >= min(q_lim[qb][qs][i], k_end)) x[i] = __float_as_uint(kNegInf);
                        }
                    };
                    auto relate = [&]() {  // scores to the references
#pragma unroll
                        for (int i = 0; i < N / 2; ++i) {
                            const float4 f = col[slot][i];
                            float t0, t1;
                            unpair(fma2(pair(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), pair(f.x, f.y), pair(f.z, f.w)), t0, t1);
                            x[2 * i] = __float_as_uint(t0);
                            x[2 * i + 1] = __float_as_uint(t1);
                        }
                    };
                    bool place = t == first;  // whether references are moved
                    load();
                    if (!place) {
                        relate();
                        float top = kNegInf;
#pragma unroll
                        for (int i = 0; i < N; i += 2)  // (NaN counts for nothing)
                            asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(__uint_as_float(x[i])), "f"(__uint_as_float(x[i + 1])));
                        place = slot_any(wg_id, top > kSlack + kLift);
                        if (__builtin_expect(place, 0)) load();
                    }
                    if (__builtin_expect(place, 0)) {
                        float most[(N + 15) / 16];
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const float m = warp_max(__uint_as_float(x[i]));
                            if ((i & 15) == 0 || lane == (i & 15)) most[i / 16] = m;
                        }
#pragma unroll
                        for (int j = 0; j < (N + 15) / 16; ++j)
                            if (lane < 16 && j * 16 + lane < N) warp_col[slot][warp & 3][j * 16 + lane] = most[j];
                        warps_meet(wg_id, 128);
                        if (wt < rows) {
                            float *c = reinterpret_cast<float *>(&col[slot][wt >> 1]) + (wt & 1);
                            float top = warp_col[slot][0][wt];
#pragma unroll
                            for (int w = 1; w < 4; ++w) top = fmaxf(top, warp_col[slot][w][wt]);
                            top *= c[0];
                            const float m = col_m[qb][slot][wt];
                            // also when the first score above -inf is met
                            const bool up = top > m + kSlack;
                            col_f[slot][wt] = up ? ex2(m - top) : 1.f;
                            if (up) {
                                col_m[qb][slot][wt] = top;
                                c[2] = kLift - top;
                            }
                        } else if (wt < kCols) {
                            col_f[slot][wt] = 1.f;
                        }
                        warps_meet(wg_id, 128);
                        if (t > first) {
                            // the product before this one is complete: then the outputs so far are scaled
                            wait_for(p_empty(slot, (count - 1) & 1), ((count - 1) >> 1) & 1, failed);
                            fence_after();
#pragma unroll 1
                            for (int c = 0; c < N; c += 8) {
                                uint32_t o[8];
                                load_columns<8>(oc + c, o);
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * col_f[slot][c + i]);
                                tmem_st8(oc + c, o);
                            }
                            tmem_wait_st();
                        }
#pragma unroll
                        for (int i = 0; i < N / 2; ++i) {
                            const float2 f = reinterpret_cast<const float2 *>(col_f[slot])[i];
                            l[i] = fma2(l[i], pair(f.x, f.y), 0);
                        }
                        relate();
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(s_empty(sb));
                    next_scores();
                    if ((g.two && !slot) || t + 1 < nt) next_scores();  // the other slot's, of this tile or the next
                    const int pb = count & 1;
                    wait_for(p_empty(slot, pb), ((count >> 1) & 1) ^ 1, failed);
                    const uint32_t to = pbuf + (slot * 2 + pb) * kPBytes + row * 128;
#pragma unroll
                    for (int c = 0; c < N; c += 8) {  // 16 bytes of the key's row
                        uint32_t p[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float t0 = ex2(__uint_as_float(x[c + 2 * i])), t1 = ex2(__uint_as_float(x[c + 2 * i + 1]));
                            l[c / 2 + i] = add2(l[c / 2 + i], pair(t0, t1));
                            p[i] = pack2<false>(t0, t1);
                        }
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((c >> 3) ^ (row & 7)) * 16)), "r"(p[0]), "r"(p[1]),
                                     "r"(p[2]), "r"(p[3])
                                     : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_full(slot, pb));
                }
                if (mine) {
#pragma unroll
                    for (int c = 0; c < N; c += 16) {
                        const float s = column_sums<(N < 16 ? N : 16)>(l + c / 2, lane);
                        if (lane < 16 && c + lane < N) warp_col[slot][warp & 3][c + lane] = s;
                    }
                }
            };
            if (rows <= 8)
                part_of(std::integral_constant<int, 8>());
            else if (rows <= 16)
                part_of(std::integral_constant<int, 16>());
            else if (rows <= 32)
                part_of(std::integral_constant<int, 32>());
            else
                part_of(std::integral_constant<int, 48>());
            // ---- end of the part: the columns' sums, then the outputs, thread = dimension
            if (mine) {
                warps_meet(wg_id, 128);
                if (wt < rows) {
                    const float s = (warp_col[slot][0][wt] + warp_col[slot][1][wt]) + (warp_col[slot][2][wt] + warp_col[slot][3][wt]);
                    col_l[qb][slot][wt] = s;
                    // weights were taken although no tile's maximum was above -inf: a NaN, or scores that a later tile brought
                    // within 2^8 of the reference that stands in until then, which is 0
                    if (col_m[qb][slot][wt] == kNegInf && s != 0.f) col_m[qb][slot][wt] = 0.f;
                }
                wait_for(o_full(slot), outs++ & 1, failed);
            }
            if (shared) {  // the slots join their sums, each for half of the rows
                warps_meet(3, 256);
                wait_for(o_full(slot ^ 1), outs_other++ & 1, failed);
            } else if (g.two || !mine) {
                ++outs_other;
            }
            if (mine) {
                fence_after();
                const int half = (rows + 1) >> 1, lo = shared && slot ? half : 0, hi = shared && !slot ? half : rows;
                float *to = four_part<D>(ws, blockIdx.x, g.t0 == 0 ? 1 : 0) + (size_t)(g.two && slot ? kCols : 0) * D;
                float *stats = four_part<D>(ws, blockIdx.x, g.t0 == 0 ? 1 : 0) + (size_t)kFourPartRows * D + (g.two && slot ? kCols : 0);
                if (wt < rows) {
                    float m = col_m[qb][slot][wt], s = col_l[qb][slot][wt], f0 = 1.f, f1 = 0.f;
                    if (shared) {
                        const float m1 = col_m[qb][slot ^ 1][wt], l1 = col_l[qb][slot ^ 1][wt], mx = fmaxf(m, m1);
                        f0 = m == mx ? 1.f : ex2(m - mx);  // equal, or both -inf: nothing to scale
                        f1 = m1 == mx ? 1.f : ex2(m1 - mx);
                        s = s * f0 + l1 * f1;
                        m = mx;
                    }
                    // a row that sees no key is 0; one that sees scores of -inf alone is 0 / 0 = NaN
                    if (g.whole) {
                        const float inv = v_scale / s;
                        f0 *= inv;
                        f1 *= inv;
                    } else if (wt >= lo && wt < hi) {
                        stats[wt] = m;
                        stats[kFourPartRows + wt] = s;
                    }
                    reinterpret_cast<float2 *>(&col[slot][0])[wt] = make_float2(f0, f1);
                }
                warps_meet(wg_id, 128);
                if (D == 128 || row < D) {  // (whole warps)
                    T *out = (T *)a.out + (((int64_t)g.begin + t_first) * a.q_heads + g.h * G) * D + row;
#pragma unroll 1
                    for (int c = lo & ~15; c < hi; c += 16) {
                        uint32_t x[16];
                        tmem_ld16(oc + c, x);
                        uint32_t y[16];
                        if (shared) tmem_ld16(o_col(slot ^ 1) + lanes + c, y);
                        tmem_wait_ld();
                        tmem_loaded<16>(x);
                        if (shared) tmem_loaded<16>(y);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int r = c + i;
                            if (r < lo || r >= hi) continue;
                            const float2 f = reinterpret_cast<const float2 *>(&col[slot][0])[r];
                            float o = __uint_as_float(x[i]) * f.x;
                            if (shared) o += __uint_as_float(y[i]) * f.y;
                            if (g.whole) {
                                const int tok = r / G;
                                if (q_lim[qb][qs][r] <= 0) o = 0.f;
                                out[((int64_t)tok * a.q_heads + (r - tok * G)) * D] = round_to<T>(o);
                            } else {
                                to[(size_t)r * D + row] = o;
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            fence_before();
            __syncwarp();
            // the other slot has read this one's outputs; the columns' factors are read
            if (shared)
                warps_meet(3, 256);
            else if (mine)
                warps_meet(wg_id, 128);
            if (lane == 0) {
                bar_arrive(o_empty(slot));
                bar_arrive(q_empty(qb));
            }
        }
    } else if (warp < 16) {
        // ------------------------------------------------------------------ codes to operands: thread = key, or value dimension
        asm volatile("setmaxnreg.dec.sync.aligned.u32 " PCG_OTHER_REGISTERS ";");
        const bool keys = warp < 12;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t stage = 0, stage_phase = 0, T0 = 0;  // T0: tiles so far
        bool ok = keys || (warp & 3) < kValueWarps;
        while (ok && walk.next(a, TQ, g)) {
            const int nt = tiles(g), k_first = first_key(g), k_end = last_key(g);
#pragma unroll 1
            for (int t = 0; t < nt; ++t, ++T0) {
                ok = __all_sync(0xffffffffu, wait_for(full_bar(stage), stage_phase, failed));
                const uint32_t buf = T0 & 1, parity = ((T0 >> 1) & 1) ^ 1;
                ok = ok && __all_sync(0xffffffffu, wait_for(keys ? k_empty(buf) : v_empty(buf), parity, failed));
                if (!ok) break;
                fence_after();
                // (small loops: in line, the two took 1,300 and 2,000 cycles a tile, out of the instruction cache)
                const uint32_t at = ring + stage * Z::kStage;
                if (keys) {
                    const uint32_t page = at + (row >> 4) * kPage;
                    uint32_t codes = page + (row & 15) * 16, to = k_col(buf) + lanes;
                    uint64_t scales;
                    if (D == 128) {
                        asm volatile("ld.shared.b64 %0, [%1];" : "=l"(scales) : "r"(page + key_scales_at(D) + (row & 15) * 8) : "memory");
                    } else {
                        uint32_t four;
                        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(four) : "r"(page + key_scales_at(D) + (row & 15) * 4) : "memory");
                        scales = four;
                    }
#pragma unroll 1
                    for (int c = 0; c < D / 64; ++c) {  // 64 dimensions, four scales
                        uint32_t w[8], s[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(w[4 * h]), "=r"(w[4 * h + 1]), "=r"(w[4 * h + 2]), "=r"(w[4 * h + 3])
                                         : "r"(codes + h * 256)
                                         : "memory");
                        widen_scales((uint32_t)scales, s);
                        scales >>= 32;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t s0 = __byte_perm(s[h], s[h], 0x1010), s1 = __byte_perm(s[h], s[h], 0x3232);
                            uint32_t r[16];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t v[4];
                                widen_codes(w[4 * h + i], v);
#pragma unroll
                                for (int j = 0; j < 4; ++j) r[i * 4 + j] = mul2(v[j], i < 2 ? s0 : s1);
                            }
                            tmem_st16(to + h * 16, r);
                        }
                        codes += 512;
                        to += 32;
                    }
                } else {
                    // The scales first, 8 a thread, as float16 to where all 16 dimensions of a group find them; those of tokens
                    // behind the part's last key, which may be anything, as 0.
                    const int left = k_end - (k_first + t * kKeys), groups = D / 16;
                    const int page_of = row / (2 * groups), in = row % (2 * groups), token = page_of * 16 + (in & 1) * 8;
                    uint32_t two[2], f[4];
                    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(two[0]), "=r"(two[1]) : "r"(at + page_of * kPage + value_scales_at(D) + in * 8) : "memory");
                    widen_scales(two[0], reinterpret_cast<uint32_t(&)[2]>(f[0]));
                    widen_scales(two[1], reinterpret_cast<uint32_t(&)[2]>(f[2]));
                    if (__builtin_expect(left < kKeys, 0)) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            f[i] = token + 2 * i >= left ? 0u : token + 2 * i + 1 >= left ? f[i] & 0xffffu : f[i];
                    }
                    const uint32_t table = scale_buf + buf * Z::kScales;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(table + (in >> 1) * (kKeys * 2) + token * 2), "r"(f[0]), "r"(f[1]),
                                 "r"(f[2]), "r"(f[3])
                                 : "memory");
                    warps_meet(4, kValueWarps * 32);
                    uint32_t codes = at + value_codes_at(D) + row * 8, scales = table + (row >> 4) * (kKeys * 2), to = v_col(buf) + lanes;
#pragma unroll 1
                    for (int h = 0; h < 4; ++h) {  // two pages
                        uint32_t r[16];
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint32_t c[2], s[8];
                            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c[0]), "=r"(c[1]) : "r"(codes + q * kPage) : "memory");
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                             : "=r"(s[4 * i]), "=r"(s[4 * i + 1]), "=r"(s[4 * i + 2]), "=r"(s[4 * i + 3])
                                             : "r"(scales + q * 32 + i * 16)
                                             : "memory");
                            }
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                uint32_t v[4];
                                widen_codes(c[i], v);
#pragma unroll
                                for (int j = 0; j < 4; ++j) r[q * 8 + i * 4 + j] = mul2(v[j], s[i * 4 + j]);
                            }
                        }
                        tmem_st16(to, r);
                        codes += 2 * kPage;
                        scales += 64;
                        to += 16;
                    }
                }
                __syncwarp();
                if (lane == 0) bar_arrive(empty_bar(stage));
                tmem_wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(keys ? k_full(buf) : v_full(buf));
                if (++stage == S) {
                    stage = 0;
                    stage_phase ^= 1;
                }
            }
        }
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 " PCG_OTHER_REGISTERS ";");
      if (warp == 16) {
        // ------------------------------------------------------------------ copies: a lane per copy looks its block up
        const int unit = min(1 << a.bs_shift, 64);  // tokens of one copy
        uint32_t it = 0, stage = 0, stage_phase = 1;
        bool ok = true;
        auto block_of = [&](const Segment &g, int t) -> int32_t {  // of the lane's copy of tile t: -1 none there, -2 zeros
            const int p = first_key(g) + t * kKeys + lane * unit;
            if (lane * unit >= kKeys || t >= tiles(g) || p >= last_key(g)) return -1;
            const int32_t block = a.block_table[(int64_t)g.b * a.max_blocks + (p >> a.bs_shift)];
            return block < 0 || block >= a.n_blocks ? -2 : block;
        };
        bool have = walk.next(a, TQ, g);
        int32_t now = -1, soon = -1;
        if (have) {
            now = block_of(g, 0);
            soon = block_of(g, 1);
        }
        while (ok && have) {
            const int nt = tiles(g), k_first = first_key(g), k_end = last_key(g);
            Segment next;
            int32_t next0 = -1, next1 = -1;
            bool more_items = false;
#pragma unroll 1
            for (int t = 0; t < nt; ++t) {
                const int32_t later = block_of(g, t + 2);  // its latency passes under the wait
                ok = __all_sync(0xffffffffu, wait_for(empty_bar(stage), stage_phase, failed));
                if (!ok) break;
                const int k0 = k_first + t * kKeys, p = k0 + lane * unit;
                const int pages = now == -1 ? 0 : min(unit, k_end - p + 15) >> 4;
                const uint32_t dst = ring + stage * Z::kStage + lane * (unit >> 4) * kPage, bytes = pages * kPage;
                const uint32_t zeros = __ballot_sync(0xffffffffu, now == -2);
                if (zeros) {
                    if (now == -2)
                        for (uint32_t i = 0; i < bytes; i += 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + i), "r"(0u) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                const uint32_t total = __reduce_add_sync(0xffffffffu, now >= 0 ? bytes : 0u);
                const uint32_t bar = full_bar(stage);
                if (elect_one()) bar_expect(bar, total);
                __syncwarp();
                const int64_t in = (p & ((1 << a.bs_shift) - 1)) >> 4;
                const uint8_t *src = (const uint8_t *)a.k + ((((int64_t)max(now, 0) * a.kv_heads + g.h) << (a.bs_shift - 4)) + in) * kPage;
                for (int c = 0; c < kKeys / unit; ++c) {
                    const uint64_t from = __shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)src, c);
                    const uint32_t n = __shfl_sync(0xffffffffu, now >= 0 ? bytes : 0u, c);
                    if (n && elect_one())
                        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                         ring + stage * Z::kStage + c * (unit >> 4) * kPage),
                                     "l"(from), "r"(n), "r"(bar)
                                     : "memory");
                    __syncwarp();
                }
                ++it;
                if (++stage == S) {
                    stage = 0;
                    stage_phase ^= 1;
                }
                if (t == 0) {  // the next item's first blocks, looked up while this one's tiles are on their way
                    more_items = walk.next(a, TQ, next);
                    if (more_items) {
                        next0 = block_of(next, 0);
                        next1 = block_of(next, 1);
                    }
                }
                now = soon;
                soon = later;
            }
            g = next;
            have = more_items;
            now = next0;
            soon = next1;
        }
        if (*failed)  // giving up: copies already asked for may still be landing
            for (uint32_t back = 1; back <= S && back <= it; ++back) bar_drain(full_bar((it - back) % S), ((it - back) / S) & 1);
    } else if (warp == 17) {
        // ------------------------------------------------------------------ scores, issued by an elected lane
        uint32_t T0 = 0, part = 0, sb = 0, s_phase = 1;  // tiles, parts; buffer and phase of the next scores
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, wait_for(bar, parity, failed)); };
        while (ok && walk.next(a, TQ, g)) {
            const Split sp = split_of(g.n, g.pair, TQ);
            const int qb = part & 1;
            // (the same in all lanes, and known to be: operands of products then stay in uniform registers)
            const int nt = __shfl_sync(0xffffffffu, tiles(g), 0), two = __shfl_sync(0xffffffffu, (int)g.two, 0);
            // N / 8 of the slots' products, in its place in the instruction descriptor
            const uint32_t n0 = __shfl_sync(0xffffffffu, (uint32_t)((sp.tq * G + 15) >> 4) << 18, 0);
            const uint32_t n1 = two ? __shfl_sync(0xffffffffu, (uint32_t)(((sp.tokens - sp.tq) * G + 15) >> 4) << 18, 0) : n0;
            wait(q_full(qb), (part >> 1) & 1);
#pragma unroll 1
            for (int t = 0; ok && t < nt; ++t) {
                const int kb = (T0 + t) & 1;
                wait(k_full(kb), ((T0 + t) >> 1) & 1);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (!two && s != (t & 1)) continue;
                    wait(s_empty(sb), s_phase);
                    if (!ok) break;
                    fence_after();
                    constexpr int kPart = (kCols * 128) >> 4;
                    const uint64_t q = desc_k(qbuf + qb * (2 * Z::kQSlot) + (two ? s : 0) * Z::kQSlot);
                    const uint32_t idesc = kIdescQK | (s ? n1 : n0);
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk)
                            mma_ts(s_col(sb), k_col(kb) + kk * 8, q + (kk >> 2) * kPart + (kk & 3) * 2, idesc, kk > 0);
                        mma_commit(s_full(sb));
                        if (s || !two) mma_commit(k_empty(kb));
                        if ((s || !two) && t == nt - 1) mma_commit(q_empty(qb));
                    }
                    __syncwarp();
                    if (++sb == kScoreBufs) {
                        sb = 0;
                        s_phase ^= 1;
                    }
                }
            }
            T0 += nt;
            ++part;
        }
        if (*failed) {  // products already issued may still be writing tensor memory: it is freed when they have retired
            if (elect_one()) mma_commit(drain);
            bar_drain(drain, 0);
        }
    } else if (warp == 19) {
        // ------------------------------------------------------------------ outputs, likewise
        uint32_t T0 = 0, part = 0, used[2] = {0, 0};  // tiles; of the slots: weights taken
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, wait_for(bar, parity, failed)); };
        while (ok && walk.next(a, TQ, g)) {
            const Split sp = split_of(g.n, g.pair, TQ);
            const int nt = __shfl_sync(0xffffffffu, tiles(g), 0), two = __shfl_sync(0xffffffffu, (int)g.two, 0), each = two ? 1 : 2;
            const uint32_t n0 = __shfl_sync(0xffffffffu, (uint32_t)((sp.tq * G + 15) >> 4) << 18, 0);
            const uint32_t n1 = two ? __shfl_sync(0xffffffffu, (uint32_t)(((sp.tokens - sp.tq) * G + 15) >> 4) << 18, 0) : n0;
#pragma unroll 1
            for (int t = 0; ok && t < nt; ++t) {
                const int vb = (T0 + t) & 1;
                wait(v_full(vb), ((T0 + t) >> 1) & 1);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (!two && s != (t & 1)) continue;
                    const int pb = used[s] & 1, begun = t >= each;
                    wait(p_full(s, pb), (used[s] >> 1) & 1);
                    if (!begun) wait(o_empty(s), (part & 1) ^ 1);
                    if (!ok) break;
                    fence_after();
                    ++used[s];
                    const uint64_t p = desc_mn(pbuf + (s * 2 + pb) * kPBytes, kKeys);
                    const uint32_t idesc = kIdescPV | (s ? n1 : n0);
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < kKeys / 16; ++kk)
                            mma_ts(o_col(s), v_col(vb) + kk * 8, p + kk * (2048 >> 4), idesc, begun || kk > 0);
                        mma_commit(p_empty(s, pb));
                        if (t + each >= nt) mma_commit(o_full(s));
                        if (s || !two) mma_commit(v_empty(vb));
                    }
                    __syncwarp();
                }
            }
            T0 += nt;
            ++part;
        }
        if (*failed) {
            if (elect_one()) mma_commit(drain + 8);
            bar_drain(drain + 8, 0);
        }
    } else {
        // ------------------------------------------------------------------ queries of the next item
        constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;  // 16 bytes a lane
        const int sub = lane / kLanes, chunk = lane % kLanes;
        bool ok = true;
        for (uint32_t part = 0; ok && walk.next(a, TQ, g); ++part) {
            const int qb = part & 1;
            const Split sp = split_of(g.n, g.pair, TQ);
            ok = __all_sync(0xffffffffu, wait_for(q_empty(qb), ((part >> 1) & 1) ^ 1, failed));
            if (!ok) break;
#pragma unroll 1
            for (int s = 0; s < (g.two ? 2 : 1); ++s) {
                const int t0 = g.pair * 2 * TQ + (s ? sp.tq : 0), rows = (s ? sp.tokens - sp.tq : sp.tq) * G, padded = (rows + 15) & ~15;
                const uint32_t to = qbuf + qb * (2 * Z::kQSlot) + s * Z::kQSlot + (chunk >> 3) * (kCols * 128);
                constexpr int kAhead = 4;  // loads in flight a lane
#pragma unroll 1
                for (int r0 = 0; r0 < padded; r0 += kAhead * kRowsAtOnce) {
                    uint4 w[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int r = r0 + i * kRowsAtOnce + sub, tok = r / G;
                        w[i] = make_uint4(0u, 0u, 0u, 0u);
                        if (r < rows)
                            w[i] = *reinterpret_cast<const uint4 *>((const T *)a.q + ((int64_t)g.begin + t0 + tok) * a.q_stride +
                                                                    ((int64_t)g.h * G + (r - tok * G)) * D + chunk * 8);
                    }
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int r = r0 + i * kRowsAtOnce + sub;
                        float by = a.scale_log2;
                        if constexpr (std::is_same<T, uint16_t>::value) {
                            // bfloat16: the row is multiplied by the power of two that brings its largest finite value to 2^14 or
                            // above, so that float16 holds it exactly down to 2^-28 of that, and to 2^-39 of it below
                            float x[8], most = 0.f;
                            Elem<uint16_t>::unpack(w[i], x);
#pragma unroll
                            for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]) < __int_as_float(0x7f800000) ? fabsf(x[j]) : 0.f);
#pragma unroll
                            for (int o = kLanes / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                            const int up = max(-113, min(120, 14 + 127 - (int)(__float_as_uint(most) >> 23)));
                            const float f = __uint_as_float((uint32_t)(127 + up) << 23);
                            by *= __uint_as_float((uint32_t)(127 - up) << 23);
                            w[i] = make_uint4(pack2<false>(x[0] * f, x[1] * f), pack2<false>(x[2] * f, x[3] * f), pack2<false>(x[4] * f, x[5] * f),
                                              pack2<false>(x[6] * f, x[7] * f));
                        }
                        if (r < padded) {
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + r * 128 + (((chunk & 7) ^ (r & 7)) * 16)), "r"(w[i].x),
                                         "r"(w[i].y), "r"(w[i].z), "r"(w[i].w)
                                         : "memory");
                            if (chunk == 0) {
                                // (never 0 for a row that is there: 0 times a masked score would be NaN)
                                q_by[qb][s][r] = r < rows ? fminf(fmaxf(by, 1.17549435e-38f), 3.40282347e38f) : 0.f;
                                q_lim[qb][s][r] = g.len - g.n + t0 + r / G + 1;
                            }
                        }
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(q_full(qb));
        }
      }
    }
    fence_before();
    __syncthreads();
    if (tid == 0) reinterpret_cast<WorkspaceHead *>(ws)->failed[blockIdx.x] = failed_flag;
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

// ---------------------------------------------------------------------------------------------- combine
// Block (c, y): the item that block c of the main kernel began and did not end, if there is one; its rows y, y + gridDim.y,
// ...; thread = dimension.  What bounds it is the latency of the parts' loads, which do not depend on each other.
constexpr int kJoinThreads = 256, kJoinBlocks = 4;

template <int D, typename T>
__global__ void __launch_bounds__(kJoinThreads) attention_fourbit_join_kernel(const __grid_constant__ AttnArgs a, float v_scale, void *ws) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const WorkspaceHead *head = reinterpret_cast<const WorkspaceHead *>(ws);
    const int tid = threadIdx.x, dim = tid % D, c = blockIdx.x;
    const Run next = head->run[c + 1];
    const int64_t begun = head->run[c].first, all = head->run[kMaxBlocks].first;
    if (__syncthreads_or(tid < kMaxBlocks && head->failed[tid])) {  // no row may pass for a result
        const uint32_t nan2 = 0x7fff7fffu;  // NaN in both types
        const int64_t vecs = (int64_t)a.rows * a.q_heads * (D * (int)sizeof(T) / 16), blocks = (int64_t)gridDim.x * gridDim.y;
        for (int64_t i = ((int64_t)blockIdx.y * gridDim.x + c) * kJoinThreads + tid; i < vecs; i += blocks * kJoinThreads)
            reinterpret_cast<uint4 *>(a.out)[i] = make_uint4(nan2, nan2, nan2, nan2);
        return;
    }
    if (next.first >= all || next.tile == 0 || next.first - next.tile < begun) return;
    const int G = a.q_heads / a.kv_heads, TQ = kCols / G;
    int begin, n, len;
    attn_sequence(a, next.b, begin, n, len);
    const int64_t end = next.first - next.tile + tiles_of(n, len, TQ, next.pair);
    int last = c + 1;  // the block that ends the item
    while (last + 1 < kMaxBlocks && head->run[last + 1].first < end) ++last;
    const Split sp = split_of(n, next.pair, TQ);
    // the first part lies among its block's parts that begin an item, the others among those that do not
    const float *first = four_part<D>(ws, c, 1), *rest = four_part<D>(ws, c + 1, 0);
    constexpr int64_t kStride = 2 * (int64_t)kFourPartRows * (D + 2), kM = (int64_t)kFourPartRows * D, kL = kM + kFourPartRows;
    const int parts = last - c;
    for (int r = blockIdx.y * (kJoinThreads / D) + tid / D; r < sp.tokens * G; r += kJoinBlocks * (kJoinThreads / D)) {
        const int tok = r / G, row = sp.two && tok >= sp.tq ? kCols + r - sp.tq * G : r;
        const float m0 = first[kM + row];
        float m = m0;
#pragma unroll 8
        for (int k = 0; k < parts; ++k) m = fmaxf(m, rest[k * kStride + kM + row]);
        float f = m0 == kNegInf ? 0.f : m0 == m ? 1.f : ex2(m0 - m);
        float l = first[kL + row] * f, o = first[(int64_t)row * D + dim] * f;
#pragma unroll 4
        for (int k = 0; k < parts; ++k) {
            const float *p = rest + k * kStride;
            const float mk = p[kM + row];
            f = mk == kNegInf ? 0.f : mk == m ? 1.f : ex2(mk - m);
            l += p[kL + row] * f;
            o += p[(int64_t)row * D + dim] * f;
        }
        const int t_row = next.pair * 2 * TQ + tok;
        const bool empty = len - n + t_row + 1 <= 0;
        ((T *)a.out)[(((int64_t)begin + t_row) * a.q_heads + next.h * G + (r - tok * G)) * D + dim] = round_to<T>(empty ? 0.f : o * (v_scale / l));
    }
}

template <int D, typename T>
cudaError_t launch(const AttnArgs &a, float v_scale, void *ws, cudaStream_t stream) {
    static std::atomic<uint64_t> prepared{0};  // devices whose kernel has been given its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev > 63 || !(prepared.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(attention_fourbit_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sizes4<D>::kSmem);
        if (e == cudaSuccess && dev <= 63) prepared.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
        e = launch_behind(attention_fourbit_kernel<D, T>, dim3(kMaxBlocks), kFourbitThreads, (size_t)Sizes4<D>::kSmem, stream, a, v_scale, ws);
    if (e == cudaSuccess)
        e = launch_behind(attention_fourbit_join_kernel<D, T>, dim3(kMaxBlocks, kJoinBlocks), kJoinThreads, 0, stream, a, v_scale, ws);
    return e;
}

}  // namespace

pcg_status attention_fourbit_tc(const char *who, const AttnArgs &a, pcg_dtype dtype, float v_scale, void *ws, cudaStream_t stream) {
    cudaError_t e;
    if (a.d == 128)
        e = dtype == PCG_BF16 ? launch<128, uint16_t>(a, v_scale, ws, stream) : launch<128, f16_t>(a, v_scale, ws, stream);
    else
        e = dtype == PCG_BF16 ? launch<64, uint16_t>(a, v_scale, ws, stream) : launch<64, f16_t>(a, v_scale, ws, stream);
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

}  // namespace pcg
