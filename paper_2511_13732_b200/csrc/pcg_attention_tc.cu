// Attention on the 5th-generation tensor cores: bfloat16 and float16, head dimensions 64 and 128.
//
// The rows of one key head -- G = q_heads / kv_heads query heads for each of a sequence's new tokens -- are packed
// token by token into tiles of 128 rows (TQ = 128 / G tokens), so that a key or value is fetched once for the heads that
// share it and a drafted chunk's few tokens fill as much of a tile as there is.  An ITEM is a (sequence, key head, pair of
// row tiles).  A block works on an item with two SLOTS, each a warpgroup with its own scores and its own output accumulator
// in tensor memory:
//   two row tiles (chunks of prompts):      key tiles of 128 keys; slot s has row tile s, and every key tile goes to both.
//                                           Bound by the products, and by the softmax between them.
//   one row tile (tokens, drafted chunks):  key tiles of 64 keys; both slots have that row tile and take the key tiles in
//                                           turn, and their sums meet at the end.  Bound by HBM: a stage of the ring waits
//                                           for its tile's softmax, so that half as large a tile leaves more of the ring
//                                           for tiles that are on their way.
// Measured (after a pause, 1.7 to 1.9 GHz): one prompt of 8192, 32 / 8 heads x 128, 502 us = 1095 TFLOP/s (65 % of the
// measured cuBLAS burst); 64 tokens over up to 8000 cached, the same heads, 197 us = 5.98 TB/s (93 % of the measured copy).
//
// attention_tc_kernel        Every block first cuts the call's work into one equal run per block, whatever the lengths are:
//                            it numbers the units of all items, one for each 64 keys and four for what an item costs
//                            beside its keys, and looks up where its own run begins and ends.  No block waits for
//                            another, and an item may be shared.  Then 8 softmax warps (two slots), a warp that fetches
//                            (TMA) and a warp that issues tcgen05.mma go through the run.  An item that a block has to
//                            itself is written out; a part of one goes to the workspace as an unscaled sum with its
//                            reference and its sum of weights.
// attention_combine_kernel   joins the parts of items that were shared, in the order of the blocks.
//
// Tensor memory: scores S0, S1 (128 columns each, fp32), outputs O0, O1 (D columns each, fp32).  The weights of a tile
// replace the scores they come from, packed to 16 bits in the first 64 columns, and are the A operand of the product with
// the values straight from there.  The next scores of a slot are issued behind that product by the same thread: the
// tensor pipe runs a block's products in the order of their issue, so the weights have been read by then, and the
// barrier that announces the new scores also says that the product before them is complete.
#include <cuda.h>  // CUtensorMap and its enums only; the encoder is fetched through the runtime, not linked
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "pcg_attention_work.cuh"

namespace pcg {

constexpr int kSoftmaxWarps = 8;
constexpr int kThreads = 32 * (kSoftmaxWarps + 2);
constexpr float kSlack = 8.f;    // the reference may lag the maximum by a factor 2^8 before sums are scaled

// ---------------------------------------------------------------------------------------------- device primitives
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Bounded wait for a phase of an mbarrier: false = gave up, or another role has.  A poll may suspend the thread for a
// time that the hardware sets (microseconds), so the limit is some tens of milliseconds at least and seconds at most.
constexpr uint32_t kPolls = 1u << 21;
__device__ __forceinline__ bool bar_poll(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
__device__ __forceinline__ bool bar_wait_hot(uint32_t bar, uint32_t parity, volatile int *failed) {
    for (uint32_t i = 0; i < kPolls; ++i) {
        if (bar_poll(bar, parity)) return true;
        if (*failed) return false;
    }
    *failed = 1;
    return false;
}
// The same with the loop out of line: there are some twenty waits, and with a loop in each the kernel's code misses the
// instruction cache more often (256 drafted chunks: 265 us, so 247).  The products for head dimension 128 keep theirs.
__device__ __noinline__ bool bar_wait_on(uint32_t bar, uint32_t parity, volatile int *failed) {
    return bar_wait_hot(bar, parity, failed);
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *failed) {
    return bar_poll(bar, parity) || bar_wait_on(bar, parity, failed);
}
// The same without a look at the failure flag: what is in flight is waited for after a failure too.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kPolls; ++i)
        if (bar_poll(bar, parity)) return;
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One lane of a converged warp, the same one every time.  The tensor-core and copy instructions take their operands from the
// warp's uniform registers: where one lane is chosen by a comparison, each of them is issued by a loop over the lanes
// (about 90 cycles an instruction), and behind this one at once.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// Arrives when all products that this thread has issued are complete.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
}
// Operand descriptors, 128-byte swizzle (layout type 2 at bit 61, version 1 at bit 46); byte offsets >> 4.
// K-major (queries and keys: rows of 64 head dimensions, 128 bytes): groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// MN-major (values: rows are keys, the product's inner index; 64 head dimensions a row): blocks of 64 head dimensions
// `keys` * 128 bytes apart (leading offset), groups of 8 keys 1024 bytes apart (stride offset).
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, int keys) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)((keys * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
}
#define PCG_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define PCG_W8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of the warp's 32 lanes; the caller waits (tmem_wait_ld / _st)
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : PCG_R8(v, 0), PCG_R8(v, 8), PCG_R8(v, 16), PCG_R8(v, 24)
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        PCG_W8(v, 0), PCG_W8(v, 8), PCG_W8(v, 16), PCG_W8(v, 24)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : PCG_R8(v, 0), PCG_R8(v, 8)
        : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        PCG_W8(v, 0), PCG_W8(v, 8)
        : "memory");
}
// Waits for the loads so far.  A load's registers are named again behind the wait, so that no use moves ahead of it.
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void tmem_loaded(uint32_t *v) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
        asm volatile("" : "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]),
                     "+r"(v[i + 7]));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Two floats in a 64-bit register pair, for the packed fp32 instructions.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// NaN if one of the three is.
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// 32 weights 2^(score * scale + shift), packed to 16 bits; their sums, in pairs.  All by the special-function unit: with
// 6, 10, 13 or 16 of 32 computed by a polynomial on the FMA pipes a prompt of 8192 tokens took 2 to 9 % longer, since a
// tile's time is the latency of its steps rather than the unit's rate.
template <bool BF16>
__device__ __forceinline__ void weights(const uint32_t *v, uint64_t scale, uint64_t shift, uint64_t (&sum)[4], uint32_t *p) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float a, b;
        unpair(fma2(pair(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), scale, shift), a, b);
        a = ex2(a);
        b = ex2(b);
        sum[i & 3] = add2(sum[i & 3], pair(a, b));
        p[i] = pack2<BF16>(a, b);
    }
}

// 32 bytes of a row (the lanes' rows are apart: whole sectors at least).
__device__ __forceinline__ void store_row(void *p, const uint32_t (&w)[8], bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), PCG_W8(w, 0) : "memory");
    } else {  // 16-byte alignment
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// ---------------------------------------------------------------------------------------------- main kernel
template <int D>
struct Sizes {
    static constexpr int kTileBytes = kTile * D * 2;         // a row tile or a key tile: D / 64 parts of 128 rows x 128 bytes
    // Ring, 160 KB: a stage holds 128 keys or their values, or 64 keys and then their values, each as D / 64 parts.
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kSmem = (2 + kStages) * kTileBytes;  // 224 KB; 3 KB are left for all else
    static_assert((2 + kStages) * kTileBytes >= kAttnMaxB * 12, "the cut's scratch");
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
    attention_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap qmap,
                        const __grid_constant__ CUtensorMap qmap_few, const __grid_constant__ CUtensorMap kmap,
                        const __grid_constant__ CUtensorMap vmap, void *ws) {
    constexpr int S = Sizes<D>::kStages, kParts = D / 64, kTileBytes = Sizes<D>::kTileBytes;
    // instruction descriptors: D = fp32, A and B of one 16-bit type, M = 128; N = 128 keys, B K-major; N = D, B MN-major
    constexpr uint32_t kType = BF16 ? (1u << 7) | (1u << 10) : 0u;
    constexpr uint32_t kIdescQK = (1u << 4) | kType | ((kTile >> 3) << 17) | ((kTile >> 4) << 24);
    constexpr uint32_t kIdescQKHalf = (1u << 4) | kType | ((kHalf >> 3) << 17) | ((kTile >> 4) << 24);  // N = 64 keys
    constexpr uint32_t kIdescPV = (1u << 4) | kType | (1u << 16) | ((D >> 3) << 17) | ((kTile >> 4) << 24);
    // float16's weights are kept 2^7 higher than the reference says, out of the range where they lose bits: 2^8 above the
    // reference is then 2^15 at most.  The sums carry the same factor, so it cancels.
    constexpr float kLift = BF16 ? 0.f : 7.f;

    extern __shared__ __align__(1024) unsigned char smem_raw[];  // swizzled tiles start on 1024-byte boundaries
    __shared__ int64_t warp_units[kThreads / 32], warp_items[kThreads / 32];
    __shared__ Run run[2];
    __shared__ __align__(8) uint64_t bars[2 * S + 15];
    __shared__ float slot_m[2][kTile], slot_l[2][kTile];  // for the end of an item with one row tile
    __shared__ uint32_t tmem_slot;
    __shared__ int failed_flag;
    volatile int *failed = &failed_flag;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t qbuf = smem_u32(smem_raw), ring = qbuf + 2 * kTileBytes, bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };         // a stage has landed
    auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };  // a stage has been read
    const uint32_t q_full = bar0 + 8u * (2 * S), q_empty = q_full + 8, drain = q_full + 16;
    auto s_full = [&](int s) { return q_full + 24u + 8u * s; };   // a slot's scores are complete
    auto p_full = [&](int s) { return q_full + 40u + 8u * s; };   // ... its weights are in place
    auto o_full = [&](int s) { return q_full + 56u + 8u * s; };   // ... its last product is complete
    auto written = [&](int s) { return q_full + 104u + 8u * s; };  // a slot's outputs of an item are out of its stage
    auto p_half = [&](int s) { return q_full + 88u + 8u * s; };   // ... those of the first 64 keys
    const uint32_t merge_full = q_full + 72, merge_done = q_full + 80;  // both slots' references and sums are there, read

    if (tid == 0) {
        for (int i = 0; i < 2 * S + 15; ++i) {
            // by a slot's warps: its weights, its outputs (4); by both slots': the hand-over (8); by one thread or the
            // hardware: all others
            const uint32_t bar = bar0 + 8u * i;
            const uint32_t count = bar == p_full(0) || bar == p_full(1) || bar >= p_half(0) ? 4 : bar >= merge_full ? 8 : 1;
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed_flag = (qbuf & 1023u) != 0;  // never: the array is declared so
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    if (tid < 3 * 32 && lane == 0)
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(warp == 0 ? &qmap_few : warp == 1 ? &kmap : &vmap)) : "memory");
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_slot;
    auto s_col = [&](int s) { return tmem + (uint32_t)(s * kTile); };
    auto o_col = [&](int s) { return tmem + (uint32_t)(2 * kTile + s * D); };
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int G = a.q_heads / a.kv_heads, TQ = kTile / G;
    cut_work(a, TQ, reinterpret_cast<int64_t *>(smem_raw), warp_units, warp_items, run);
    // In a long run, rows of the first queries' tile that no item with one row tile loads are zero: the products of padding
    // then cost little power, which the clock of a call bound by HBM depends on (64 tokens over 8000, call after call at
    // 1000 W: 247 -> 227 us).
    if (run[1].first - run[0].first >= 64) {
        for (int i = tid; i < kTileBytes / 16; i += kThreads) reinterpret_cast<uint4 *>(smem_raw)[i] = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    if (tid == 0) reinterpret_cast<WorkspaceHead *>(ws)->run[blockIdx.x] = run[0];
    if (tid == 0 && blockIdx.x == kMaxBlocks - 1) reinterpret_cast<WorkspaceHead *>(ws)->run[kMaxBlocks] = run[1];
    Walk walk;
    walk.start(a, run[0], run[1]);
    Segment g;
    if (warp < kSoftmaxWarps) {
        // ------------------------------------------------------------------ softmax: thread = row of the slot's row tile
        const int slot = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t sc = s_col(slot) + lanes, oc = o_col(slot) + lanes;
        const int tok = row / G, head = row - tok * G;
        uint32_t sn = 0, on = 0, on_other = 0, mn = 0, wn = 0;  // phases met so far
        uint32_t loads = 0;                             // stages filled so far
        bool ok = true;
        while (ok && walk.next(a, TQ, g)) {
            const int t_row = g.pair * 2 * TQ + (g.two ? slot * TQ : 0) + tok;  // the row's token in its sequence
            const bool valid = tok < TQ && t_row < g.n;
            const int lim = valid ? g.len - g.n + t_row + 1 : 0x7fffffff;  // padding rows never ask for masking
            const bool warp_valid = __any_sync(0xffffffffu, valid);
            const int first = g.two ? 0 : slot, step = g.two ? 1 : 2;
            float m = kNegInf, l = 0.f;
            bool bad = false;
            for (int t = first; t < g.nt; t += step, ++sn) {
                ok = __all_sync(0xffffffffu, bar_wait(s_full(slot), sn & 1, failed));
                if (!ok) break;
                fence_after();
                const int keys = g.two ? kTile : kHalf, k0 = (g.t0 + t) * keys;
                if (t == g.nt - 1 && k0 + keys > g.len && (!g.two || slot == 0)) {
                    // Values behind the sequence's last token may hold anything, and 0 * NaN is NaN: they are zeroed
                    // where they lie.  This stage is the last of the part; the slot's weights are announced after it, and
                    // slot 1's product comes behind slot 0's.
                    const uint32_t i = loads + (g.two ? 2 * g.nt : g.nt) - 1;
                    ok = __all_sync(0xffffffffu, bar_wait(full_bar(i % S), (i / S) & 1, failed));
                    if (!ok) break;
                    if (row < keys && k0 + row >= g.len) {
                        const uint32_t at = ring + (i % S) * kTileBytes + (g.two ? 0 : kTileBytes / 2) + row * 128;
#pragma unroll 1
                        for (int part = 0; part < kParts; ++part)
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + part * (keys * 128) + c * 16), "r"(0u)
                                             : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (warp_valid) {
                    uint32_t v[64];
                    float top[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
                    if (__any_sync(0xffffffffu, lim < k0 + keys)) {
                        // Scores of keys that a row does not see become -inf where they lie, 16 columns at a time: first those
                        // that some of the warp's rows see, then those that none does.  (In line, over all columns, this took
                        // 2,000 cycles: code that runs once an item comes at some 6 cycles an instruction, being out of the
                        // instruction cache.  So does all else that an item has once, hence the small loops below.)
                        const int seen = max(lim - k0, 0);
                        int c = __reduce_min_sync(0xffffffffu, seen) & ~15;
                        const int none = __reduce_max_sync(0xffffffffu, valid ? seen : 0);
                        uint32_t x[16];
#pragma unroll 1
                        for (; c < none && c < keys; c += 16) {
                            tmem_ld16(sc + c, x);
                            tmem_wait_ld();
                            tmem_loaded<16>(x);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (c + i >= seen) x[i] = __float_as_uint(kNegInf);
                            tmem_st16(sc + c, x);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(kNegInf);
#pragma unroll 1
                        for (; c < keys; c += 16) tmem_st16(sc + c, x);
                        tmem_wait_st();
                    }
                    auto take_max = [&](const uint32_t (&x)[64]) {
#pragma unroll
                        for (int c = 0; c < 64; c += 2)
                            top[(c >> 1) & 3] = max3_nan(top[(c >> 1) & 3], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
                    };
                    tmem_ld32(sc, v);
                    tmem_ld32(sc + 32, v + 32);
                    if (g.two) {
                        uint32_t u[64];
                        tmem_ld32(sc + 64, u);
                        tmem_ld32(sc + 96, u + 32);
                        tmem_wait_ld();
                        tmem_loaded<64>(u);
                        take_max(u);
                    } else {
                        tmem_wait_ld();
                    }
                    tmem_loaded<64>(v);
                    take_max(v);
                    const float mt = max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]) * a.scale_log2;
                    bad = bad || !(mt < -kNegInf);
                    // also when the first score above -inf is met; a row's reference depends on its own scores alone, and
                    // padding rows, whose scores are arbitrary, have none
                    const bool move = valid && mt > m + kSlack;
                    if (__any_sync(0xffffffffu, move)) {
                        const float mnew = move ? mt : m, f = move ? ex2(m - mt) : 1.f;
                        l *= f;
                        if (t > first) {
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(oc + c, o);
                                tmem_wait_ld();
                                tmem_loaded<16>(o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st16(oc + c, o);
                            }
                        }
                        m = mnew;
                    }
                    // a row that has met no score above -inf yet weighs everything 0
                    const float by = !valid ? kNegInf : (m == kNegInf ? 0.f : -m) + kLift;  // (padding: 0 too)
                    const uint64_t scale2 = pair(a.scale_log2, a.scale_log2), by2 = pair(by, by);
                    uint64_t sum[4] = {0, 0, 0, 0};
                    // Half the keys at a time: the product with the first half's values starts while the other weights are
                    // computed.  The second half's scores are read again, into the registers that the first half leaves: a
                    // loop of two turns keeps the code in the instruction cache, which 128 scores in line do not fit.  (The
                    // first half's weights lie where its own scores were.)
#pragma unroll 1
                    for (int h = 0; h < (g.two ? 2 : 1); ++h) {
                        uint32_t p[32];
                        if (h) {
                            tmem_wait_ld();
                            tmem_loaded<64>(v);
                        }
                        weights<BF16>(v, scale2, by2, sum, p);
                        if (!h && g.two) tmem_ld32(sc + 64, v);
                        weights<BF16>(v + 32, scale2, by2, sum, p + 16);
                        if (!h && g.two) tmem_ld32(sc + 96, v + 32);
                        tmem_st32(sc + h * 32, p);
                        tmem_wait_st();
                        if (!h && g.two) {
                            fence_before();
                            __syncwarp();
                            if (lane == 0) bar_arrive(p_half(slot));
                        }
                    }
                    float s0, s1;
                    unpair(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
                    l += s0 + s1;
                } else if (g.two) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_half(slot));
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full(slot));
            }
            if (bad) l = __int_as_float(0x7fffffff);  // a score of +inf or NaN
            if (!ok) break;
            loads += g.two ? 2 * g.nt : g.nt;
            // ---- end of the part
            const bool mine = first < g.nt;                    // this slot has had a key tile
            const bool shared = !g.two && g.nt > 1;            // both have, of one row tile
            if (mine) ok = __all_sync(0xffffffffu, bar_wait(o_full(slot), on++ & 1, failed));
            if (!ok) break;
            if (shared) {  // the slots join their sums, each for one half of the head dimensions
                slot_m[slot][row] = m;
                slot_l[slot][row] = l;
                __syncwarp();
                if (lane == 0) bar_arrive(merge_full);
                ok = __all_sync(0xffffffffu, bar_wait(merge_full, mn & 1, failed)) &&
                     __all_sync(0xffffffffu, bar_wait(o_full(slot ^ 1), on_other++ & 1, failed));
                if (!ok) break;
            } else if (g.two || !mine) {
                ++on_other;
            }
            // With two row tiles, outputs are staged in the item's last two stages of the ring (slot 0 in the keys', slot 1 in
            // the values'), which the products leave to the softmax to release: all that read them is complete.
            const uint32_t last = (loads - (slot == 0 ? 2 : 1)) % S, staged = ring + last * kTileBytes;
            if (mine) {
                fence_after();
                if (warp_valid) {
                    float f0 = 1.f, f1 = 0.f;
                    if (shared) {
                        const float m1 = slot_m[slot ^ 1][row], l1 = slot_l[slot ^ 1][row], mx = fmaxf(m, m1);
                        f0 = m == mx ? 1.f : ex2(m - mx);  // equal, or both -inf: nothing to scale
                        f1 = m1 == mx ? 1.f : ex2(m1 - mx);
                        l = l * f0 + l1 * f1;
                        m = mx;
                    }
                    // a row that sees no key is 0 (below); one that sees scores of -inf alone is 0 / 0 = NaN
                    if (g.whole) {
                        const float inv = 1.f / l;
                        f0 *= inv;
                        f1 *= inv;
                    }
                    const int prow = (g.two ? slot * kTile : 0) + row;
                    float *part = part_base(ws, blockIdx.x, g.t0 == 0 ? 1 : 0, D);
                    const uint32_t stage_row = staged + row * (D * 2);
                    const int64_t offset = valid ? (((int64_t)g.begin + t_row) * a.q_heads + g.h * G + head) * (D * 2) : -1;
                    const bool wide = ((uintptr_t)a.out & 31) == 0;
#pragma unroll 1
                    for (int c = shared && slot ? D / 2 : 0; c < (shared && !slot ? D / 2 : D); c += 16) {
                        uint32_t o[16];
                        tmem_ld16(oc + c, o);
                        if (shared) {
                            uint32_t o1[16];
                            tmem_ld16(o_col(slot ^ 1) + lanes + c, o1);
                            tmem_wait_ld();
                            tmem_loaded<16>(o);
                            tmem_loaded<16>(o1);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + __uint_as_float(o1[i]) * f1);
                        } else {
                            tmem_wait_ld();
                            tmem_loaded<16>(o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f0);
                        }
                        if (g.whole) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                w[j] = lim <= 0 ? 0u : pack2<BF16>(__uint_as_float(o[2 * j]), __uint_as_float(o[2 * j + 1]));
                            if (g.two) {
                                // 16-byte chunks of the row, permuted by its number: a warp's lanes meet all banks alike
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage_row + (((c >> 3) + i) ^ (row & 7)) * 16),
                                                 "r"(w[4 * i]), "r"(w[4 * i + 1]), "r"(w[4 * i + 2]), "r"(w[4 * i + 3])
                                                 : "memory");
                            } else if (valid) {  // few rows: straight to memory
                                store_row((char *)a.out + offset + c * 2, w, wide);
                            }
                        } else if (valid) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) part[(size_t)(c + i) * kPartRows + prow] = __uint_as_float(o[i]);
                        }
                        __syncwarp();  // the next columns are read by the whole warp
                    }
                    if (valid && !g.whole && !(shared && slot)) {
                        part[(size_t)D * kPartRows + prow] = m;
                        part[(size_t)(D + 1) * kPartRows + prow] = l;
                    }
                    if (g.whole && g.two) {
                        // whole rows to memory, 32 / (D / 8) at a time: a row a lane would touch 32 lines a store, which took
                        // 4,400 cycles a tile of head dimension 128
                        constexpr int kChunks = D / 8, kRowsAtOnce = 32 / kChunks;
                        const int rows = 32 - __clz(__ballot_sync(0xffffffffu, valid));  // valid rows come first
                        const int chunk = lane % kChunks;
                        const uint32_t stage_warp = staged + (warp & 3) * 32 * (D * 2);
#pragma unroll 1
                        for (int r0 = 0; r0 < rows; r0 += 4 * kRowsAtOnce) {
                            uint32_t w[4][4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int r = (r0 + k * kRowsAtOnce + lane / kChunks) & 31;
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                             : "=r"(w[k][0]), "=r"(w[k][1]), "=r"(w[k][2]), "=r"(w[k][3])
                                             : "r"(stage_warp + r * (D * 2) + (chunk ^ (r & 7)) * 16)
                                             : "memory");
                            }
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int r = r0 + k * kRowsAtOnce + lane / kChunks;
                                const int64_t to = __shfl_sync(0xffffffffu, offset, r & 31);
                                if (r < rows && to >= 0)
                                    *reinterpret_cast<uint4 *>((char *)a.out + to + chunk * 16) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
                            }
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // copies land there next
                    }
                }
                fence_before();
                __syncwarp();
                if (g.two) {
                    if (lane == 0) bar_arrive(written(slot));
                    if ((warp & 3) == 0) {  // the stage is free when all four warps are through
                        ok = __all_sync(0xffffffffu, bar_wait(written(slot), wn & 1, failed));
                        if (ok && lane == 0) bar_arrive(empty_bar(last));
                    }
                    ++wn;
                } else if (shared) {  // the other slot has read this one's sums
                    if (lane == 0) bar_arrive(merge_done);
                    ok = __all_sync(0xffffffffu, bar_wait(merge_done, mn++ & 1, failed));
                }
            }
        }
    } else if (warp == kSoftmaxWarps) {
        // ------------------------------------------------------------------ fetch: a lane per page looks its block up, one issues
        const bool paged = a.kv_len != nullptr;
        const int box = paged ? min(1 << a.bs_shift, kHalf) : kHalf;  // rows of one copy
        const uint32_t few = a.few_tokens, few_rows = few * G;
        uint32_t it = 0, stage = 0, stage_phase = 1, items = 0;  // a stage's first fill waits for nothing: parity 1 has passed
        bool ok = true;
        auto page_of = [&](const Segment &g, int t) -> int32_t {  // the block of key tile t's rows from lane * box on
            const int p = (g.t0 + t) * (g.two ? kTile : kHalf) + lane * box;
            if (!paged || lane >= 8 || t >= g.nt || p >= g.len) return -1;
            const int32_t block = a.block_table[(int64_t)g.b * a.max_blocks + (p >> a.bs_shift)];
            return block < 0 || block >= a.n_blocks ? a.n_blocks : block;  // behind the tensor: reads zeros
        };
        bool have = walk.next(a, TQ, g);
        int32_t page0 = -1, page1 = -1, page2 = -1;  // blocks of the tiles t .. t + 2
        if (have) {
            page0 = page_of(g, 0);
            page1 = page_of(g, 1);
            page2 = page_of(g, 2);
        }
        while (ok && have) {
            // the queries: G heads of TQ tokens at a time, which is the row tile's order
            if (items > 0) ok = __all_sync(0xffffffffu, bar_wait(q_empty, (items - 1) & 1, failed));
            if (!ok) break;
            ++items;
            if (elect_one()) {
                // two row tiles, or the tokens of one, `few` at a time; all in one where the last copy would end behind the tile
                const uint32_t tokens = g.n - g.pair * 2 * TQ, few_copies = (tokens + few - 1) / few;
                const bool all = g.two || few_copies * few_rows > kTile;
                const uint32_t rows = all ? G * TQ : few_rows, step = g.two ? kTile : few_rows, copies = g.two ? 2 : all ? 1 : few_copies;
                bar_expect(q_full, copies * rows * kParts * 128);
#pragma unroll 1
                for (uint32_t c = 0; c < copies; ++c)
#pragma unroll
                    for (int part = 0; part < kParts; ++part)  // (the second row tile's parts lie behind the first's)
                        tma_load(qbuf + part * (kTile * 128) + c * step * 128 * (g.two ? kParts : 1), all ? &qmap : &qmap_few, part * 64, 0,
                                 g.h, g.begin + g.pair * 2 * TQ + c * (all ? TQ : few), q_full);
            }
            __syncwarp();
            // Two row tiles: the keys of tile 0, its values, the keys of tile 1, and so on, a stage each.  One: the keys and
            // values of a tile in one stage.
            Segment next;
            int32_t next0 = -1, next1 = -1, next2 = -1;
            const int loads = g.two ? 2 * g.nt : g.nt;
#pragma unroll 1
            for (int j = 0; j < loads; ++j) {
                const int t = g.two ? j >> 1 : j, keys = g.two ? kTile : kHalf, k0 = (g.t0 + t) * keys;
                const uint32_t s = stage;
                const int32_t page3 = page_of(g, t + 3);  // its latency passes under the wait
                ok = __all_sync(0xffffffffu, bar_wait(empty_bar(s), stage_phase, failed));
                if (!ok) break;
                if (++stage == S) {
                    stage = 0;
                    stage_phase ^= 1;
                }
                ++it;
                // rows behind the sequence's pages are not fetched: their scores are masked, their values zeroed
                const int copies = min(keys / box, (max(g.len - k0, 0) + box - 1) / box);
                const CUtensorMap *map = g.two && (j & 1) ? &vmap : &kmap;
                const uint32_t bar = full_bar(s);
                int c0 = 0;
#pragma unroll 1
                do {  // (four at a time: small blocks' copies are paced by their issue)
                    int32_t block[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) block[c] = paged ? __shfl_sync(0xffffffffu, page0, c0 + c) : 0;
                    if (elect_one()) {
                        if (c0 == 0) bar_expect(bar, copies * box * (g.two ? 1 : 2) * D * 2);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (c0 + c >= copies) break;
                            const uint32_t dst = ring + s * kTileBytes + (c0 + c) * box * 128;
                            const int r = k0 + (c0 + c) * box;
                            const int c1 = paged ? r & ((1 << a.bs_shift) - 1) : g.h, c2 = paged ? g.h : g.begin + r;
#pragma unroll
                            for (int part = 0; part < kParts; ++part) {
                                tma_load(dst + part * (keys * 128), map, part * 64, c1, c2, block[c], bar);
                                if (!g.two)
                                    tma_load(dst + kTileBytes / 2 + part * (keys * 128), &vmap, part * 64, c1, c2, block[c], bar);
                            }
                        }
                    }
                    __syncwarp();
                    c0 += 4;
                } while (c0 < copies);
                if (j == 0) {  // the next item's lengths and first blocks, looked up while this one's tiles are on their way
                    have = walk.next(a, TQ, next);
                    if (have) {
                        next0 = page_of(next, 0);
                        next1 = page_of(next, 1);
                        next2 = page_of(next, 2);
                    }
                }
                if (!g.two || (j & 1)) {
                    page0 = page1;
                    page1 = page2;
                    page2 = page3;
                }
            }
            g = next;
            page0 = next0;
            page1 = next1;
            page2 = next2;
        }
        if (*failed) {  // giving up: copies already asked for may still be landing
            if (items > 0) bar_drain(q_full, (items - 1) & 1);
            for (uint32_t back = 1; back <= S && back <= it; ++back) bar_drain(full_bar((it - back) % S), ((it - back) / S) & 1);
        }
    } else {
        // ------------------------------------------------------------------ products
        // Head dimension 128: one lane, elected once, waits and issues, which costs the fewest instructions between two
        // products (a prompt of 8192: 525 us with the warp waiting and a lane elected for each issue, 512 so).  64: the warp
        // waits (16 prompts of up to 1500: 101 us with one lane, 95 so: its code is the smaller).
        constexpr bool kOneLane = D == 128;
        auto issuing = [&]() { return kOneLane || elect_one(); };
        auto together = [&]() {
            if (!kOneLane) __syncwarp();
        };
        if (!kOneLane || elect_one()) {
            // stages in the order of their use, weights of a slot and queries: number (of a stage) and phase of the next
            uint32_t stage = 0, stage_phase = 0, h_phase = 0, p_phase0 = 0, p_phase1 = 0, q_phase = 0;
            bool ok = true;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (kOneLane)
                    ok = ok && bar_wait_hot(bar, parity, failed);
                else
                    ok = ok && __all_sync(0xffffffffu, bar_wait(bar, parity, failed));
            };
            auto next_stage = [&]() {  // waits for it
                const uint32_t s = stage;
                wait(full_bar(s), stage_phase);
                if (++stage == S) {
                    stage = 0;
                    stage_phase ^= 1;
                }
                return s;
            };
            const uint64_t qdesc = desc_k(qbuf), kdesc = desc_k(ring);
            const uint64_t vdesc = desc_mn(ring, kTile), vdesc_half = desc_mn(ring + kTileBytes / 2, kHalf);
            constexpr uint32_t kStep = kTileBytes >> 4;
            // All by the elected lane.  A slot's scores of 128 or 64 keys; 64 keys' weights, from column col on, with their values.
            auto scores = [&](int slot, uint64_t q, uint32_t s) {
                constexpr int kPart = (kTile * 128) >> 4;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(s_col(slot), q + (kk >> 2) * kPart + (kk & 3) * 2, kdesc + s * kStep + (kk >> 2) * kPart + (kk & 3) * 2, kIdescQK, kk > 0);
                mma_commit(s_full(slot));
            };
            auto scores_half = [&](int slot, uint32_t s) {
                constexpr int kPart = (kTile * 128) >> 4, kPartK = (kHalf * 128) >> 4;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(s_col(slot), qdesc + (kk >> 2) * kPart + (kk & 3) * 2, kdesc + s * kStep + (kk >> 2) * kPartK + (kk & 3) * 2, kIdescQKHalf,
                           kk > 0);
                mma_commit(s_full(slot));
            };
            auto outputs = [&](int slot, int col, uint64_t v, bool begun) {
#pragma unroll
                for (int kk = 0; kk < kHalf / 16; ++kk)
                    mma_ts(o_col(slot), s_col(slot) + col + kk * 8, v + kk * (2048 >> 4), kIdescPV, begun || kk > 0);
            };
            while (ok && walk.next(a, TQ, g)) {
                wait(q_full, q_phase);
                q_phase ^= 1;
                if (g.two) {
                    const uint32_t s = next_stage();
                    if (!ok) break;
                    fence_after();
                    for (int slot = 0; slot < 2; ++slot)
                        if (issuing()) scores(slot, qdesc + slot * kStep, s);
                    if (issuing()) mma_commit(g.nt == 1 ? q_empty : empty_bar(s));  // (the last keys' stage is the softmax's)
                    together();
                    for (int t = 0; ok && t < g.nt; ++t) {
                        const uint32_t vs = next_stage();
                        const bool more = t + 1 < g.nt;
                        uint32_t ks = 0;
                        if (!ok) break;
                        // each slot in turn: its weights with the values of stage vs, in two halves, then the scores of its next
                        // key tile
#pragma unroll
                        for (int slot = 0; slot < 2; ++slot) {
                            wait(p_half(slot), h_phase);
                            if (!ok) break;
                            fence_after();
                            const uint64_t v = vdesc + vs * kStep;
                            if (issuing()) outputs(slot, 0, v, t > 0);
                            together();
                            if (more && slot == 0) ks = next_stage();
                            wait(p_full(slot), slot ? p_phase1 : p_phase0);
                            if (!ok) break;
                            fence_after();
                            if (issuing()) {
                                outputs(slot, 32, v + 4 * (2048 >> 4), true);
                                if (more) {
                                    scores(slot, qdesc + slot * kStep, ks);
                                    if (slot) mma_commit(t + 2 == g.nt ? q_empty : empty_bar(ks));
                                } else {
                                    mma_commit(o_full(slot));
                                }
                                if (slot && more) mma_commit(empty_bar(vs));
                            }
                            together();
                        }
                        h_phase ^= 1;
                        p_phase0 ^= 1;
                        p_phase1 ^= 1;
                    }
                } else {
                    uint32_t mine[2] = {0, 0};  // the stages of the slots' key tiles
                    for (int t = 0; ok && t < g.nt + 2; ++t) {
                        // tile t - 2's weights with its values; then tile t's scores, in the same slot
                        const int slot = t & 1;
                        if (t >= 2) {
                            wait(p_full(slot), slot ? p_phase1 : p_phase0);
                            if (slot)
                                p_phase1 ^= 1;
                            else
                                p_phase0 ^= 1;
                            if (!ok) break;
                            fence_after();
                            const uint32_t s = slot ? mine[1] : mine[0];
                            if (issuing()) {
                                outputs(slot, 0, vdesc_half + s * kStep, t >= 4);
                                mma_commit(empty_bar(s));
                                if (t >= g.nt) mma_commit(o_full(slot));
                            }
                            together();
                        } else if (t >= g.nt) {
                            continue;  // one key tile: the other slot has none
                        }
                        if (t < g.nt) {
                            const uint32_t s = next_stage();
                            if (!ok) break;
                            fence_after();
                            if (slot)
                                mine[1] = s;
                            else
                                mine[0] = s;
                            if (issuing()) {
                                scores_half(slot, s);
                                if (t == g.nt - 1) mma_commit(q_empty);
                            }
                            together();
                        }
                    }
                }
            }
            if (*failed) {  // products already issued may still be writing tensor memory: it is freed when they have retired
                together();
                if (issuing()) mma_commit(drain);
                together();
                bar_drain(drain, 0);
            }
            }
    }
    fence_before();
    __syncthreads();
    if (tid == 0) reinterpret_cast<WorkspaceHead *>(ws)->failed[blockIdx.x] = failed_flag;
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

// ---------------------------------------------------------------------------------------------- host
namespace {

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
    static const EncodeTiled fn = []() -> EncodeTiled {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// Rank 4, 64 elements (128 bytes, swizzled) of the innermost dimension a copy; what lies outside reads as zero.
CUresult encode(CUtensorMap *map, bool bf16, const void *p, const cuuint64_t (&dim)[4], const cuuint64_t (&stride)[3],
                const cuuint32_t (&box)[4]) {
    const cuuint32_t one[4] = {1u, 1u, 1u, 1u};
    return encoder()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void *>(p),
                     dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// Tokens of one copy of an item with one row tile: about a sixteenth of a row tile, in whole groups of 8 rows (the swizzle's
// period).
int few_tokens(int G, int TQ) {
    const int group = G % 8 == 0 ? 1 : G % 4 == 0 ? 2 : G % 2 == 0 ? 4 : 8, want = (TQ / 16 + group - 1) / group * group;
    return want < group ? group : want;
}

template <int D, bool BF16>
cudaError_t launch(const AttnArgs &a, const CUtensorMap &q, const CUtensorMap &few, const CUtensorMap &k, const CUtensorMap &v, void *ws, cudaStream_t stream) {
    static std::atomic<uint64_t> prepared{0};  // devices whose kernel has been given its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev > 63 || !(prepared.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(attention_tc_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sizes<D>::kSmem);
        if (e == cudaSuccess && dev <= 63) prepared.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
        e = launch_behind(attention_tc_kernel<D, BF16>, dim3(kMaxBlocks), kThreads, (size_t)Sizes<D>::kSmem, stream, a, q, few, k, v, ws);
    if (e == cudaSuccess)
        e = launch_behind(attention_combine_kernel<D, typename std::conditional<BF16, uint16_t, f16_t>::type>, dim3(kMaxBlocks, kCombineDims, kCombineRows), kCombineThreads, 0, stream, a, ws);
    return e;
}

}  // namespace

size_t attention_work_bytes(int32_t d) {
    return (kHeadBytes + (size_t)kMaxBlocks * 2 * kPartRows * (d + 2) * 4 + 255) / 256 * 256;
}

pcg_status attention_tc(const char *who, const AttnArgs &args, pcg_dtype dtype, void *workspace, cudaStream_t stream) {
    if (!encoder()) {
        set_error("%s: the driver does not provide cuTensorMapEncodeTiled", who);
        return PCG_ERR_CUDA;
    }
    const bool bf16 = dtype == PCG_BF16;
    AttnArgs a = args;
    a.few_tokens = few_tokens(a.q_heads / a.kv_heads, kTile / (a.q_heads / a.kv_heads));
    const cuuint64_t d = a.d, G = a.q_heads / a.kv_heads, heads = a.kv_heads, rows = a.rows;
    const cuuint32_t g = (cuuint32_t)G, tokens = (cuuint32_t)(kTile / G);
    alignas(64) CUtensorMap q, few, k, v;
    CUresult r = encode(&q, bf16, a.q, {d, G, heads, rows}, {d * 2, G * d * 2, (cuuint64_t)a.q_stride * 2}, {64u, g, 1u, tokens});
    if (r == CUDA_SUCCESS)
        r = encode(&few, bf16, a.q, {d, G, heads, rows}, {d * 2, G * d * 2, (cuuint64_t)a.q_stride * 2},
                   {64u, g, 1u, (cuuint32_t)a.few_tokens});
    if (a.kv_len) {
        const cuuint64_t bs = 1ull << a.bs_shift, blocks = a.n_blocks;
        const cuuint32_t box = bs < kHalf ? (cuuint32_t)bs : kHalf;
        if (r == CUDA_SUCCESS) r = encode(&k, bf16, a.k, {d, bs, heads, blocks}, {d * 2, bs * d * 2, heads * bs * d * 2}, {64u, box, 1u, 1u});
        if (r == CUDA_SUCCESS) r = encode(&v, bf16, a.v, {d, bs, heads, blocks}, {d * 2, bs * d * 2, heads * bs * d * 2}, {64u, box, 1u, 1u});
    } else {
        const cuuint64_t ks = (cuuint64_t)a.k_stride * 2, vs = (cuuint64_t)a.v_stride * 2;
        if (r == CUDA_SUCCESS) r = encode(&k, bf16, a.k, {d, heads, rows, 1}, {d * 2, ks, rows * ks}, {64u, 1u, kHalf, 1u});
        if (r == CUDA_SUCCESS) r = encode(&v, bf16, a.v, {d, heads, rows, 1}, {d * 2, vs, rows * vs}, {64u, 1u, kHalf, 1u});
    }
    if (r != CUDA_SUCCESS) {
        set_error("%s: cuTensorMapEncodeTiled failed (%d)", who, (int)r);
        return PCG_ERR_CUDA;
    }
    cudaError_t e;
    if (a.d == 128)
        e = bf16 ? launch<128, true>(a, q, few, k, v, workspace, stream) : launch<128, false>(a, q, few, k, v, workspace, stream);
    else
        e = bf16 ? launch<64, true>(a, q, few, k, v, workspace, stream) : launch<64, false>(a, q, few, k, v, workspace, stream);
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

}  // namespace pcg
