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
#include "pcg_fourbit.cuh"
#include "pcg_tcgen05.cuh"

namespace pcg {

constexpr int kSoftmaxWarps = 8;
constexpr int kThreads = 32 * (kSoftmaxWarps + 2);
// Over the cache that holds 4.5 bits a value: 8 warps between the fetch and the products round queries and widen codes to float16
// tiles.  640 threads are launched with 96 registers each, 480 for the five warps of each quarter of an SM, whose registers are its
// own: the softmax's two take 144, which the other three leave by keeping 64 (2 * 144 + 3 * 64 = 480).  Two of the 20 warps have
// no part; without them, 18 would be launched with 96 as well and have less to share.
// Measured: 2 chunks of 2048 over 16,000, 32 / 8 heads x 128, 1077 us = 1061 TFLOP/s (65 % of the measured burst); 256 chunks of
// 17 over up to 2000, 270 us, where HBM would allow 62.  What bounds those: an item's ends (14 items a block) and the hand-overs of
// a key tile from copy to widening, products, softmax and products, some 3,500 cycles a tile.
constexpr int kWidenWarps = 8, kFourbitThreads = 32 * (kSoftmaxWarps + kWidenWarps + 4);
// What an item costs there (256 chunks of 17: 306 us with four units, 288 with six, 292 with eight; 32 of 64 over 500: 76, 69, 67 with nine).
constexpr int kFourbitItemUnits = 6;
constexpr int kLaunchRegisters = 96, kSoftmaxRegisters = 144, kOtherRegisters = 64;
static_assert(2 * kSoftmaxRegisters + 3 * kOtherRegisters <= 5 * kLaunchRegisters, "the wait for more than there are would not end");
constexpr float kSlack = 8.f;    // the reference may lag the maximum by a factor 2^8 before sums are scaled

// 32 weights 2^(score * scale + shift), packed to 16 bits; their sums, in pairs, in float32 and of the weights before the rounding.
// (16 bits are what the product with the values takes, of the values' type: float16 over 4 bits, whatever the queries are.)  All by the special-function unit: with
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
template <int D, bool FOUR, int P>
struct Sizes {
    static constexpr int kTileBytes = kTile * D * 2;         // a row tile or a key tile: D / 64 parts of 128 rows x 128 bytes
    // Tiles of queries: two, one row tile each, or an item's in turn; over 4 bits and with one row tile an item one, which leaves the
    // ring a stage more (256 chunks of 17: 292 us, so 278: the next item's queries come behind this one's last values anyway).
    static constexpr int kQueryTiles = FOUR ? P : 2;
    // Ring, 160 KB: a stage holds 128 keys or their values, or 64 keys and then their values, each as D / 64 parts.
    // (4 bits: 96 or 128 KB; the codes of a tile's keys and values lie in one of three stages before it.  With half of those
    // a copy's latency showed: 256 chunks of 17, 375 us, so 343.)
    static constexpr int kStages = FOUR ? (D == 128 ? 5 : 10) - kQueryTiles : D == 128 ? 5 : 10;
    static constexpr int kCodeStages = FOUR ? (D == 128 ? 3 : 6) : 0, kCodeBytes = 8 * page_bytes(D);
    static constexpr int kSmem = (kQueryTiles + kStages) * kTileBytes + kCodeStages * kCodeBytes;  // 214 or 224 KB; 3 KB are left for all else
    static_assert(kSmem >= kAttnMaxB * 12, "the cut's scratch");
};

// FOUR: over the cache that holds 4.5 bits a value.  Operands are float16 whatever the queries' type: codes times scales have six
// significant bits, bfloat16 queries are multiplied by a power of two, a row's own, that brings them into range.  Values are
// K-major there (a dimension's keys together, as the codes are): parts of D rows of 64 keys.
template <int D, bool BF16, bool FOUR, int P>
__global__ void __launch_bounds__(FOUR ? kFourbitThreads : kThreads, 1)
    attention_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap qmap,
                        const __grid_constant__ CUtensorMap qmap_few, const __grid_constant__ CUtensorMap kmap,
                        const __grid_constant__ CUtensorMap vmap, void *ws) {
    using Z = Sizes<D, FOUR, P>;
    constexpr int S = Z::kStages, kParts = D / 64, kTileBytes = Z::kTileBytes, U = Z::kCodeStages, kAll = FOUR ? kFourbitThreads : kThreads;
    constexpr bool kWide = BF16 && !FOUR;  // bfloat16 operands
    // instruction descriptors: D = fp32, A and B of one 16-bit type, M = 128; N = 128 keys, B K-major; N = D, B MN-major
    constexpr uint32_t kType = kWide ? (1u << 7) | (1u << 10) : 0u;
    constexpr uint32_t kIdescQK = (1u << 4) | kType | ((kTile >> 3) << 17) | ((kTile >> 4) << 24);
    constexpr uint32_t kIdescQKHalf = (1u << 4) | kType | ((kHalf >> 3) << 17) | ((kTile >> 4) << 24);  // N = 64 keys
    constexpr uint32_t kIdescPV = (1u << 4) | kType | (FOUR ? 0u : 1u << 16) | ((D >> 3) << 17) | ((kTile >> 4) << 24);
    // float16's weights are kept 2^7 higher than the reference says, out of the range where they lose bits: 2^8 above the
    // reference is then 2^15 at most.  The sums carry the same factor, so it cancels.
    constexpr float kLift = kWide ? 0.f : 7.f;

    extern __shared__ __align__(1024) unsigned char smem_raw[];  // swizzled tiles start on 1024-byte boundaries
    __shared__ int64_t warp_units[kAll / 32], warp_items[kAll / 32];
    __shared__ Run run[2];
    __shared__ __align__(8) uint64_t bars[2 * S + 15 + (FOUR ? 2 * U + 4 : 0)];
    __shared__ float q_by[FOUR ? 2 : 1][FOUR ? kTile : 1];  // (4 bits) of the rows of the queries' two tiles: what scores are multiplied by
    __shared__ float slot_m[2][kTile], slot_l[2][kTile];  // for the end of an item with one row tile
    __shared__ uint32_t tmem_slot;
    __shared__ int failed_flag;
    volatile int *failed = &failed_flag;
    auto wait_on = [&](uint32_t bar, uint32_t parity, volatile int *failed) {
        if constexpr (FOUR)
            return bar_wait_small(bar, parity, failed);
        else
            return bar_wait(bar, parity, failed);
    };
    auto wait_hot = [](uint32_t bar, uint32_t parity, volatile int *failed) {
        if constexpr (FOUR)
            return bar_wait_small(bar, parity, failed);
        else
            return bar_wait_hot(bar, parity, failed);
    };
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t qbuf = smem_u32(smem_raw), ring = qbuf + Z::kQueryTiles * kTileBytes, bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };         // a stage has landed
    auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };  // a stage has been read
    const uint32_t q_full = bar0 + 8u * (2 * S), q_empty = q_full + 8, drain = q_full + 16;
    auto s_full = [&](int s) { return q_full + 24u + 8u * s; };   // a slot's scores are complete
    auto p_full = [&](int s) { return q_full + 40u + 8u * s; };   // ... its weights are in place
    auto o_full = [&](int s) { return q_full + 56u + 8u * s; };   // ... its last product is complete
    auto written = [&](int s) { return q_full + 104u + 8u * s; };  // a slot's outputs of an item are out of its stage
    auto p_half = [&](int s) { return q_full + 88u + 8u * s; };   // ... those of the first 64 keys
    const uint32_t merge_full = q_full + 72, merge_done = q_full + 80;  // both slots' references and sums are there, read
    // 4 bits: the queries' tiles have barriers each (an item with one row tile takes one of two in turn); the codes of a tile have
    // landed, been read
    auto tile_full = [&](int i) { return q_full + 120u + 8u * i; };
    auto tile_empty = [&](int i) { return q_full + 136u + 8u * i; };
    auto code_full = [&](int i) { return q_full + 152u + 8u * i; };
    auto code_empty = [&](int i) { return q_full + 152u + 8u * (U + i); };
    const uint32_t codes = ring + S * kTileBytes;

    if (tid == 0) {
        for (int i = 0; i < 2 * S + 15 + (FOUR ? 2 * U + 4 : 0); ++i) {
            // by a slot's warps: its weights, its outputs (4); by both slots': the hand-over (8); by one thread or the
            // hardware: all others
            const uint32_t bar = bar0 + 8u * i;
            uint32_t count = bar == p_full(0) || bar == p_full(1) || bar >= p_half(0) ? 4 : bar >= merge_full ? 8 : 1;
            if constexpr (FOUR) {  // stages, and codes read: by the warps that widen; a tile of queries read: by the softmax and products
                if (bar < empty_bar(0) || bar >= code_empty(0)) count = kWidenWarps;
                if (bar >= tile_full(0) && bar < code_empty(0)) count = bar < tile_empty(0) ? kWidenWarps : bar < code_full(0) ? kSoftmaxWarps + 1 : 1;
            }
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed_flag = (qbuf & 1023u) != 0;  // never: the array is declared so
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    if (!FOUR && tid < 3 * 32 && lane == 0)
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
    cut_work<FOUR ? kFourbitItemUnits : kItemUnits, kLeast, P>(a, TQ, reinterpret_cast<int64_t *>(smem_raw), warp_units, warp_items, run);
    // In a long run, rows of the first queries' tile that no item with one row tile loads are zero: the products of padding
    // then cost little power, which the clock of a call bound by HBM depends on (64 tokens over 8000, call after call at
    // 1000 W: 247 -> 227 us).
    if (run[1].first - run[0].first >= 64) {
        for (int i = tid; i < kTileBytes / 16; i += kAll) reinterpret_cast<uint4 *>(smem_raw)[i] = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    if (tid == 0) reinterpret_cast<WorkspaceHead *>(ws)->run[blockIdx.x] = run[0];
    if (tid == 0 && blockIdx.x == kMaxBlocks - 1) reinterpret_cast<WorkspaceHead *>(ws)->run[kMaxBlocks] = run[1];
    Walk walk;
    walk.start(a, run[0], run[1]);
    Segment g;
    // 4 bits: a warp's walk rests in shared memory between items.  (In registers it drove others out to local memory, which lies
    // behind the L2 where shared memory has the L1: some 1,600 cycles a tile.)
    __shared__ Walk rest[FOUR ? kAll / 32 : 1];
    if (FOUR && lane == 0) rest[warp] = walk;
    __syncwarp();
    auto advance = [&](Segment &g, bool alone = false) {  // alone: by one lane
        if constexpr (FOUR) {
            Walk w = rest[warp];
            if (!alone) __syncwarp();
            const bool more = w.next<P>(a, TQ, g);
            if (alone || lane == 0) rest[warp] = w;
            if (!alone) __syncwarp();
            return more;
        } else {
            return walk.next<P>(a, TQ, g);
        }
    };
    // 4 bits: key tiles of 128 keys for one row tile too (HBM does not bound those items, a tile's latency does), which may end
    // behind the part's last key.
    auto two = [](const Segment &g) { return P == 2 && g.two; };
    auto big = [&](const Segment &g) { return FOUR || two(g); };
    auto tiles = [&](const Segment &g) { return FOUR && !two(g) ? (g.nt + 1) >> 1 : g.nt; };
    auto first_key = [&](const Segment &g, int t) { return FOUR && !two(g) ? g.t0 * kHalf + t * kTile : (g.t0 + t) * (two(g) ? kTile : kHalf); };
    auto last_key = [&](const Segment &g) { return two(g) ? g.len : min(g.len, (g.t0 + g.nt) * kHalf); };
    if (warp < kSoftmaxWarps) {
        // ------------------------------------------------------------------ softmax: thread = row of the slot's row tile
        if (FOUR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegisters));
        uint32_t q_used = 0, q_turn = 0;  // (4 bits) uses of the queries' tiles so far (16 bits each), the next to take
        const int slot = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t sc = s_col(slot) + lanes, oc = o_col(slot) + lanes;
        const int tok = row / G, head = row - tok * G;
        uint32_t sn = 0, on = 0, on_other = 0, mn = 0, wn = 0;  // phases met so far
        uint32_t loads = 0;                             // stages filled so far
        bool ok = true;
        while (ok && advance(g)) {
            const int t_row = g.pair * P * TQ + (two(g) ? slot * TQ : 0) + tok;  // the row's token in its sequence
            const bool valid = tok < TQ && t_row < g.n;
            const int lim = valid ? g.len - g.n + t_row + 1 : 0x7fffffff;  // padding rows never ask for masking
            const int nt = tiles(g), sees = FOUR && valid ? min(lim, last_key(g)) : lim;  // keys of this part that the row sees
            const bool warp_valid = __any_sync(0xffffffffu, valid);
            const int first = two(g) ? 0 : slot, step = two(g) ? 1 : 2;
            float by_score = a.scale_log2;
            if constexpr (FOUR) {
                const uint32_t tile = two(g) ? slot : q_turn, other = tile ^ 1;
                ok = __all_sync(0xffffffffu, wait_on(tile_full(tile), q_used >> (16 * tile) & 1, failed));
                // The other slot's tile is read there, but its turn has to have begun before this warp says that it is through with
                // it: while the other slot is behind, in an item without a key tile for it, the arrival would count for that one.
                if (two(g)) ok = ok && __all_sync(0xffffffffu, wait_on(tile_full(other), q_used >> (16 * other) & 1, failed));
                if (!ok) break;
                by_score = valid ? q_by[tile][row] : 0.f;
                __syncwarp();
                if (lane == 0) bar_arrive(tile_empty(tile));
                if (two(g) && lane == 0) bar_arrive(tile_empty(other));
                q_used += two(g) ? 0x10001u : 1u << (16 * tile);
                q_used &= 0xff00ffu;
                if (!two(g)) q_turn ^= Z::kQueryTiles - 1;
            }
            float m = kNegInf, l = 0.f;
            bool bad = false;
            for (int t = first; t < nt; t += step, ++sn) {
                ok = __all_sync(0xffffffffu, wait_on(s_full(slot), sn & 1, failed));
                if (!ok) break;
                fence_after();
                const int keys = big(g) ? kTile : kHalf, k0 = first_key(g, t);
                if (!FOUR && t == g.nt - 1 && k0 + keys > g.len && (!two(g) || slot == 0)) {
                    // Values behind the sequence's last token may hold anything, and 0 * NaN is NaN: they are zeroed
                    // where they lie.  This stage is the last of the part; the slot's weights are announced after it, and
                    // slot 1's product comes behind slot 0's.
                    const uint32_t i = loads + (two(g) ? 2 * g.nt : g.nt) - 1;
                    ok = __all_sync(0xffffffffu, wait_on(full_bar(i % S), (i / S) & 1, failed));
                    if (!ok) break;
                    if (row < keys && k0 + row >= g.len) {
                        const uint32_t at = ring + (i % S) * kTileBytes + (two(g) ? 0 : kTileBytes / 2) + row * 128;
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
                    if (__any_sync(0xffffffffu, sees < k0 + keys)) {
                        // Scores of keys that a row does not see become -inf where they lie, 16 columns at a time: first those
                        // that some of the warp's rows see, then those that none does.  (In line, over all columns, this took
                        // 2,000 cycles: code that runs once an item comes at some 6 cycles an instruction, being out of the
                        // instruction cache.  So does all else that an item has once, hence the small loops below.)
                        const int seen = max(sees - k0, 0);
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
                    auto take_max = [&](const auto &x) {
                        constexpr int kCount = (int)std::extent<typename std::remove_reference<decltype(x)>::type>::value;
#pragma unroll
                        for (int c = 0; c < kCount; c += 2)
                            top[(c >> 1) & 3] = max3_nan(top[(c >> 1) & 3], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
                    };
                    tmem_ld32(sc, v);
                    tmem_ld32(sc + 32, v + 32);
                    if (big(g)) {
                        if constexpr (FOUR) {  // 32 at a time: there are fewer registers
#pragma unroll 1
                            for (int c = 64; c < 128; c += 32) {
                                uint32_t u[32];
                                tmem_ld32(sc + c, u);
                                tmem_wait_ld();
                                tmem_loaded<32>(u);
                                take_max(u);
                            }
                        } else {
                            uint32_t u[64];
                            tmem_ld32(sc + 64, u);
                            tmem_ld32(sc + 96, u + 32);
                            tmem_wait_ld();
                            tmem_loaded<64>(u);
                            take_max(u);
                        }
                    } else {
                        tmem_wait_ld();
                    }
                    tmem_loaded<64>(v);
                    take_max(v);
                    const float mt = max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]) * by_score;
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
                    const uint64_t scale2 = pair(by_score, by_score), by2 = pair(by, by);
                    uint64_t sum[4] = {0, 0, 0, 0};
                    // Half the keys at a time: the product with the first half's values starts while the other weights are
                    // computed.  The second half's scores are read again, into the registers that the first half leaves: a
                    // loop of two turns keeps the code in the instruction cache, which 128 scores in line do not fit.  (The
                    // first half's weights lie where its own scores were.)
#pragma unroll 1
                    for (int h = 0; h < (big(g) ? 2 : 1); ++h) {
                        uint32_t p[32];
                        if (h) {
                            tmem_wait_ld();
                            tmem_loaded<64>(v);
                        }
                        weights<kWide>(v, scale2, by2, sum, p);
                        if (!h && big(g)) tmem_ld32(sc + 64, v);
                        weights<kWide>(v + 32, scale2, by2, sum, p + 16);
                        if (!h && big(g)) tmem_ld32(sc + 96, v + 32);
                        tmem_st32(sc + h * 32, p);
                        tmem_wait_st();
                        if (!h && big(g)) {
                            fence_before();
                            __syncwarp();
                            if (lane == 0) bar_arrive(p_half(slot));
                        }
                    }
                    float s0, s1;
                    unpair(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
                    l += s0 + s1;
                } else if (big(g)) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_half(slot));
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_full(slot));
            }
            if (bad) l = __int_as_float(0x7fffffff);  // a score of +inf or NaN
            if (!ok) break;
            loads += big(g) ? 2 * nt : nt;
            // ---- end of the part
            const bool mine = first < nt;                    // this slot has had a key tile
            const bool shared = !two(g) && nt > 1;            // both have, of one row tile
            if (mine) ok = __all_sync(0xffffffffu, wait_on(o_full(slot), on++ & 1, failed));
            if (!ok) break;
            if (shared) {  // the slots join their sums, each for one half of the head dimensions
                slot_m[slot][row] = m;
                slot_l[slot][row] = l;
                __syncwarp();
                if (lane == 0) bar_arrive(merge_full);
                ok = __all_sync(0xffffffffu, wait_on(merge_full, mn & 1, failed)) &&
                     __all_sync(0xffffffffu, wait_on(o_full(slot ^ 1), on_other++ & 1, failed));
                if (!ok) break;
            } else if (two(g) || !mine) {
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
                        const float inv = (FOUR ? a.v_scale : 1.f) / l;
                        f0 *= inv;
                        f1 *= inv;
                    }
                    const int prow = (two(g) ? slot * kTile : 0) + row;
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
                            if (two(g)) {
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
                    if (g.whole && two(g)) {
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
                if (two(g)) {
                    if (lane == 0) bar_arrive(written(slot));
                    if ((warp & 3) == 0) {  // the stage is free when all four warps are through
                        ok = __all_sync(0xffffffffu, wait_on(written(slot), wn & 1, failed));
                        if (ok && lane == 0) bar_arrive(empty_bar(last));
                    }
                    ++wn;
                } else if (shared) {  // the other slot has read this one's sums
                    if (lane == 0) bar_arrive(merge_done);
                    ok = __all_sync(0xffffffffu, wait_on(merge_done, mn++ & 1, failed));
                }
            }
        }
    } else if (FOUR && warp < kSoftmaxWarps + kWidenWarps) {
        // ------------------------------------------------------------------ (4 bits) codes to tiles, by all eight warps each
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        const int w = tid - 32 * kSoftmaxWarps;
        uint32_t stage = 0, stage_phase = 1, unit = 0, unit_phase = 0;
        bool ok = true;
        // (each in two steps, all loads first: they are not moved ahead of stores)
        constexpr int N = 2;
        // 16 N dimensions from d0 on of key number `key` of the tile, whose page starts at `page`
        auto widen_key = [&](uint32_t tile, uint32_t page, int key, int d0) {
            const int tok = key & 15;
            uint32_t c[N][2], both;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int d = d0 + 16 * n;
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c[n][0]), "=r"(c[n][1]) : "r"(page + (d >> 5) * 256 + tok * 16 + (d & 16) / 2) : "memory");
            }
            uint32_t s[2];
            asm volatile("{\n\t.reg .u16 t;\n\tld.shared.u16 t, [%1];\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(both) : "r"(page + key_scales_at(D) + tok * (D / 16) + d0 / 16) : "memory");
            widen_scales(both, s);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int d = d0 + 16 * n;
                uint32_t r[8];
                const uint32_t by = __byte_perm(s[0], s[0], n & 1 ? 0x3232 : 0x1010);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t v[4];
                    widen_codes(c[n][i], v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) r[i * 4 + j] = mul_f16x2(v[j], by);
                }
                const uint32_t to = tile + (d >> 6) * (kTile * 128) + key * 128;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((((d & 63) >> 3) + i) ^ (key & 7)) * 16), "r"(r[4 * i]),
                                 "r"(r[4 * i + 1]), "r"(r[4 * i + 2]), "r"(r[4 * i + 3])
                                 : "memory");
            }
        };
        // 16 N values of dimension `dim`, from token k of the tile at `code` on; `left` tokens of the tile there are (the scales of
        // others may be anything: 0)
        auto widen_value = [&](uint32_t part, uint32_t code, int dim, int k, int left) {
            uint32_t c[N][2], x[N][4];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t page = code + ((k >> 4) + n) * page_bytes(D);
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c[n][0]), "=r"(c[n][1]) : "r"(page + value_codes_at(D) + dim * 8) : "memory");
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(x[n][0]), "=r"(x[n][1]), "=r"(x[n][2]), "=r"(x[n][3])
                             : "r"(page + value_scales_at(D) + (dim & ~15))
                             : "memory");
            }
            if (__builtin_expect(left < k + 16 * N, 0)) {
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int there = left - k - 16 * n - 4 * i;
                        x[n][i] = there >= 4 ? x[n][i] : there <= 0 ? 0u : x[n][i] & ((1u << (8 * there)) - 1);
                    }
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                uint32_t s[8], r[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) widen_scales(x[n][i], reinterpret_cast<uint32_t(&)[2]>(s[2 * i]));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t v[4];
                    widen_codes(c[n][i], v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) r[i * 4 + j] = mul_f16x2(v[j], s[i * 4 + j]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(part + dim * 128 + ((((k & 63) >> 3) + 2 * n + i) ^ (dim & 7)) * 16), "r"(r[4 * i]),
                                 "r"(r[4 * i + 1]), "r"(r[4 * i + 2]), "r"(r[4 * i + 3])
                                 : "memory");
            }
        };
        auto arrive = [&](uint32_t bar) {
            __syncwarp();
            if (lane == 0) bar_arrive(bar);
        };
        uint32_t used = 0, turn = 0;  // uses of the queries' tiles so far (16 bits each), the next to take
        // An item's queries, rounded to float16.  (Two warps of their own, an item ahead, were too slow for two row tiles, which
        // cannot be fetched ahead, by some 20 us an item, and for short contexts; for others this costs the same.)
        auto queries = [&](const Segment &g) {
            constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;  // 16 bytes a lane
            constexpr int kAhead = 2;  // loads in flight (256 chunks of 17: 270 us, with one 286, with four, which spread fewer rows over the warps, 278)
            const int sub = lane / kLanes, chunk = lane % kLanes;
            const uint32_t one_of = (65536 + G - 1) / G;  // r / G is r * one_of >> 16, for r < 128
            const int tokens = min(g.n - g.pair * P * TQ, P * TQ);
#pragma unroll 1
            for (int x = 0; x < (two(g) ? 2 : 1); ++x) {
                const uint32_t tile = two(g) ? x : turn;
                if (!__all_sync(0xffffffffu, wait_on(tile_empty(tile), (used >> (16 * tile) & 1) ^ 1, failed))) return false;
                const int t0 = g.pair * P * TQ + x * TQ, rows = min(tokens - x * TQ, TQ) * G;
                const uint32_t to = qbuf + tile * kTileBytes + (chunk >> 3) * (kTile * 128);
#pragma unroll 1
                for (int r0 = (warp - kSoftmaxWarps) * kAhead * kRowsAtOnce; r0 < rows; r0 += kWidenWarps * kAhead * kRowsAtOnce) {
                    uint4 v[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int r = r0 + i * kRowsAtOnce + sub, tok = r * one_of >> 16;
                        v[i] = make_uint4(0u, 0u, 0u, 0u);
                        if (r < rows)
                            v[i] = *reinterpret_cast<const uint4 *>((const uint16_t *)a.q + ((int64_t)g.begin + t0 + tok) * a.q_stride +
                                                                    ((int64_t)g.h * G + (r - tok * G)) * D + chunk * 8);
                    }
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int r = r0 + i * kRowsAtOnce + sub;
                        const float by = BF16 ? narrow_row<kLanes>(reinterpret_cast<uint4(&)[1]>(v[i])) * a.scale_log2 : a.scale_log2;
                        if (r < rows) {
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + r * 128 + ((chunk & 7) ^ (r & 7)) * 16), "r"(v[i].x),
                                         "r"(v[i].y), "r"(v[i].z), "r"(v[i].w)
                                         : "memory");
                            // (never 0: 0 times a masked score would be NaN)
                            if (chunk == 0) q_by[tile][r] = fminf(fmaxf(by, 1.17549435e-38f), 3.40282347e38f);
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(tile_full(tile));
                used += 1u << (16 * tile);
                used &= 0xff00ffu;
            }
            if (!two(g)) turn ^= Z::kQueryTiles - 1;
            return true;
        };
        while (ok && advance(g)) {
            const int loads = 2 * tiles(g);
            ok = queries(g);
            if (!ok) break;
#pragma unroll 1
            for (int j = 0; j < loads; ++j) {  // the keys of a tile, its values
                const int t = j >> 1;
                ok = __all_sync(0xffffffffu, wait_on(empty_bar(stage), stage_phase, failed));
                ok = ok && __all_sync(0xffffffffu, wait_on(code_full(unit), unit_phase, failed));
                if (!ok) break;
                const uint32_t tile = ring + stage * kTileBytes, code = codes + unit * Z::kCodeBytes;
                if (!(j & 1)) {  // a key, half of its dimensions a thread
                    const int key = w & (kTile - 1), d0 = w / kTile * (D / 2);
#pragma unroll 1
                    for (int d = d0; d < d0 + D / 2; d += 32) widen_key(tile, code + (key >> 4) * page_bytes(D), key, d);
                } else {  // a dimension, D / 2 of the tile's keys a thread
                    const int dim = w & (D - 1), first = w / D * (D / 2), left = last_key(g) - first_key(g, t);
#pragma unroll 1
                    for (int k = first; k < first + D / 2; k += 32) widen_value(tile + (k >> 6) * (D * 128), code, dim, k, left);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                arrive(full_bar(stage));
                if (j & 1) {  // the codes have been read
                    if (lane == 0) bar_arrive(code_empty(unit));
                    if (++unit == U) {
                        unit = 0;
                        unit_phase ^= 1;
                    }
                }
                if (++stage == S) {
                    stage = 0;
                    stage_phase ^= 1;
                }
            }
        }
    } else if (FOUR && warp >= kSoftmaxWarps + kWidenWarps + 2) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
    } else if (FOUR && warp == kSoftmaxWarps + kWidenWarps) {
        // ------------------------------------------------------------------ (4 bits) copies of a tile's pages: a lane per copy looks its block up
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        const int size = min(1 << a.bs_shift, 64);  // tokens of one copy
        constexpr int kPage = page_bytes(D);
        uint32_t it = 0, unit = 0, phase = 1;
        bool ok = true;
        auto block_of = [&](const Segment &g, int t) -> int32_t {  // of the lane's copy of tile t: -1 none there, -2 zeros
            const int p = first_key(g, t) + lane * size;
            if (lane * size >= kTile || t >= tiles(g) || p >= last_key(g)) return -1;
            const int32_t block = a.block_table[(int64_t)g.b * a.max_blocks + (p >> a.bs_shift)];
            return block < 0 || block >= a.n_blocks ? -2 : block;
        };
        bool have = advance(g);
        int32_t now = -1, soon = -1;
        if (have) {
            now = block_of(g, 0);
            soon = block_of(g, 1);
        }
        const uint32_t step = (size >> 4) * kPage;
        while (ok && have) {
            Segment next;
            int32_t next0 = -1, next1 = -1;
            bool more = false;
            const int count = tiles(g);
#pragma unroll 1
            for (int t = 0; t < count; ++t) {
                const int32_t later = block_of(g, t + 2);  // its latency passes under the wait
                const int p = first_key(g, t) + lane * size;
                const uint32_t bytes = now == -1 ? 0 : (min(size, last_key(g) - p + 15) >> 4) * kPage;
                const uint32_t there = now >= 0 ? bytes : 0, total = __reduce_add_sync(0xffffffffu, there);
                const int64_t in = (p & ((1 << a.bs_shift) - 1)) >> 4;
                const uint8_t *src = (const uint8_t *)a.k + ((((int64_t)max(now, 0) * a.kv_heads + g.h) << (a.bs_shift - 4)) + in) * kPage;
                const uint32_t dst = codes + unit * Z::kCodeBytes, bar = code_full(unit);
                ok = __all_sync(0xffffffffu, wait_on(code_empty(unit), phase, failed));
                if (!ok) break;
                if (__any_sync(0xffffffffu, now == -2)) {
                    if (now == -2)
                        for (uint32_t i = 0; i < bytes; i += 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + lane * step + i), "r"(0u) : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();  // (the arrival below is one lane's, and lets all lanes' zeros be read)
                }
                if (elect_one()) bar_expect(bar, total);
                __syncwarp();
#pragma unroll 1
                for (int c = 0; c < kTile / size; ++c) {
                    const uint64_t from = __shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)src, c);
                    const uint32_t n = __shfl_sync(0xffffffffu, there, c);
                    if (n && elect_one())
                        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + c * step), "l"(from),
                                     "r"(n), "r"(bar)
                                     : "memory");
                    __syncwarp();
                }
                ++it;
                if (++unit == U) {
                    unit = 0;
                    phase ^= 1;
                }
                if (t == 0) {  // the next item's first blocks, looked up while this one's tiles are on their way
                    more = advance(next);
                    if (more) {
                        next0 = block_of(next, 0);
                        next1 = block_of(next, 1);
                    }
                }
                now = soon;
                soon = later;
            }
            g = next;
            have = more;
            now = next0;
            soon = next1;
        }
        if (*failed)  // giving up: copies already asked for may still be landing
            for (uint32_t back = 1; back <= U && back <= it; ++back) bar_drain(code_full((it - back) % max(U, 1)), ((it - back) / max(U, 1)) & 1);
    } else if (!FOUR && warp == kSoftmaxWarps) {
        // ------------------------------------------------------------------ fetch: a lane per page looks its block up, one issues
        const bool paged = a.kv_len != nullptr;
        const int box = paged ? min(1 << a.bs_shift, kHalf) : kHalf;  // rows of one copy
        const uint32_t few = a.few_tokens, few_rows = few * G;
        uint32_t it = 0, stage = 0, stage_phase = 1, items = 0;  // a stage's first fill waits for nothing: parity 1 has passed
        bool ok = true;
        auto page_of = [&](const Segment &g, int t) -> int32_t {  // the block of key tile t's rows from lane * box on
            const int p = (g.t0 + t) * (two(g) ? kTile : kHalf) + lane * box;
            if (!paged || lane >= 8 || t >= g.nt || p >= g.len) return -1;
            const int32_t block = a.block_table[(int64_t)g.b * a.max_blocks + (p >> a.bs_shift)];
            return block < 0 || block >= a.n_blocks ? a.n_blocks : block;  // behind the tensor: reads zeros
        };
        bool have = advance(g);
        int32_t page0 = -1, page1 = -1, page2 = -1;  // blocks of the tiles t .. t + 2
        if (have) {
            page0 = page_of(g, 0);
            page1 = page_of(g, 1);
            page2 = page_of(g, 2);
        }
        while (ok && have) {
            // the queries: G heads of TQ tokens at a time, which is the row tile's order
            if (items > 0) ok = __all_sync(0xffffffffu, wait_on(q_empty, (items - 1) & 1, failed));
            if (!ok) break;
            ++items;
            if (elect_one()) {
                // two row tiles, or the tokens of one, `few` at a time; all in one where the last copy would end behind the tile
                const uint32_t tokens = g.n - g.pair * P * TQ, few_copies = (tokens + few - 1) / few;
                const bool all = two(g) || few_copies * few_rows > kTile;
                const uint32_t rows = all ? G * TQ : few_rows, step = two(g) ? kTile : few_rows, copies = two(g) ? 2 : all ? 1 : few_copies;
                bar_expect(q_full, copies * rows * kParts * 128);
#pragma unroll 1
                for (uint32_t c = 0; c < copies; ++c)
#pragma unroll
                    for (int part = 0; part < kParts; ++part)  // (the second row tile's parts lie behind the first's)
                        tma_load(qbuf + part * (kTile * 128) + c * step * 128 * (two(g) ? kParts : 1), all ? &qmap : &qmap_few, part * 64, 0,
                                 g.h, g.begin + g.pair * P * TQ + c * (all ? TQ : few), q_full);
            }
            __syncwarp();
            // Two row tiles: the keys of tile 0, its values, the keys of tile 1, and so on, a stage each.  One: the keys and
            // values of a tile in one stage.
            Segment next;
            int32_t next0 = -1, next1 = -1, next2 = -1;
            const int loads = two(g) ? 2 * g.nt : g.nt;
#pragma unroll 1
            for (int j = 0; j < loads; ++j) {
                const int t = two(g) ? j >> 1 : j, keys = two(g) ? kTile : kHalf, k0 = (g.t0 + t) * keys;
                const uint32_t s = stage;
                const int32_t page3 = page_of(g, t + 3);  // its latency passes under the wait
                ok = __all_sync(0xffffffffu, wait_on(empty_bar(s), stage_phase, failed));
                if (!ok) break;
                if (++stage == S) {
                    stage = 0;
                    stage_phase ^= 1;
                }
                ++it;
                // rows behind the sequence's pages are not fetched: their scores are masked, their values zeroed
                const int copies = min(keys / box, (max(g.len - k0, 0) + box - 1) / box);
                const CUtensorMap *map = two(g) && (j & 1) ? &vmap : &kmap;
                const uint32_t bar = full_bar(s);
                int c0 = 0;
#pragma unroll 1
                do {  // (four at a time: small blocks' copies are paced by their issue)
                    int32_t block[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) block[c] = paged ? __shfl_sync(0xffffffffu, page0, c0 + c) : 0;
                    if (elect_one()) {
                        if (c0 == 0) bar_expect(bar, copies * box * (two(g) ? 1 : 2) * D * 2);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (c0 + c >= copies) break;
                            const uint32_t dst = ring + s * kTileBytes + (c0 + c) * box * 128;
                            const int r = k0 + (c0 + c) * box;
                            const int c1 = paged ? r & ((1 << a.bs_shift) - 1) : g.h, c2 = paged ? g.h : g.begin + r;
#pragma unroll
                            for (int part = 0; part < kParts; ++part) {
                                tma_load(dst + part * (keys * 128), map, part * 64, c1, c2, block[c], bar);
                                if (!two(g))
                                    tma_load(dst + kTileBytes / 2 + part * (keys * 128), &vmap, part * 64, c1, c2, block[c], bar);
                            }
                        }
                    }
                    __syncwarp();
                    c0 += 4;
                } while (c0 < copies);
                if (j == 0) {  // the next item's lengths and first blocks, looked up while this one's tiles are on their way
                    have = advance(next);
                    if (have) {
                        next0 = page_of(next, 0);
                        next1 = page_of(next, 1);
                        next2 = page_of(next, 2);
                    }
                }
                if (!two(g) || (j & 1)) {
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
        if (FOUR) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        constexpr bool kOneLane = D == 128 && (!FOUR || P == 1);
        auto issuing = [&]() { return kOneLane || elect_one(); };
        auto together = [&]() {
            if (!kOneLane) __syncwarp();
        };
        if (!kOneLane || elect_one()) {
            // stages in the order of their use, weights of a slot and queries: number (of a stage) and phase of the next
            uint32_t stage = 0, stage_phase = 0, h_phase = 0, p_phase0 = 0, p_phase1 = 0, q_phase = 0;
            uint32_t q_used = 0, q_turn = 0;  // (4 bits) as the softmax's
            bool ok = true;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (kOneLane)
                    ok = ok && wait_hot(bar, parity, failed);
                else
                    ok = ok && __all_sync(0xffffffffu, wait_on(bar, parity, failed));
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
            const uint64_t vdesc = FOUR ? kdesc : desc_mn(ring, kTile), vdesc_half = FOUR ? desc_k(ring + kTileBytes / 2) : desc_mn(ring + kTileBytes / 2, kHalf);
            constexpr uint32_t kValueStep = FOUR ? 2 : 2048 >> 4, kValueHalf = FOUR ? (D * 128) >> 4 : 4 * (2048 >> 4);  // 16 keys, 64
            constexpr uint32_t kStep = kTileBytes >> 4;
            // All by the elected lane.  A slot's scores of 128 or 64 keys; 64 keys' weights, from column col on, with their values.
            auto scores = [&](int slot, uint64_t q, uint32_t s) {
                constexpr int kPart = (kTile * 128) >> 4;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(s_col(slot), q + (kk >> 2) * kPart + (kk & 3) * 2, kdesc + s * kStep + (kk >> 2) * kPart + (kk & 3) * 2, kIdescQK, kk > 0);
                mma_commit(s_full(slot));
            };
            auto scores_half = [&](int slot, uint32_t s, uint64_t q) {
                constexpr int kPart = (kTile * 128) >> 4, kPartK = (kHalf * 128) >> 4;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(s_col(slot), q + (kk >> 2) * kPart + (kk & 3) * 2, kdesc + s * kStep + (kk >> 2) * kPartK + (kk & 3) * 2, kIdescQKHalf,
                           kk > 0);
                mma_commit(s_full(slot));
            };
            auto outputs = [&](int slot, int col, uint64_t v, bool begun) {
#pragma unroll
                for (int kk = 0; kk < kHalf / 16; ++kk)
                    mma_ts(o_col(slot), s_col(slot) + col + kk * 8, v + kk * kValueStep, kIdescPV, begun || kk > 0);
            };
            uint32_t halves = 0;  // (4 bits) the slots' first halves of weights met so far
            while (ok && advance(g, kOneLane)) {
                uint32_t q_tile = 0;
                if constexpr (FOUR) {
                    q_tile = two(g) ? 0 : q_turn;
                    wait(tile_full(q_tile), q_used >> (16 * q_tile) & 1);
                    if (two(g)) wait(tile_full(1), q_used >> 16 & 1);
                    q_used = (q_used + (two(g) ? 0x10001u : 1u << (16 * q_tile))) & 0xff00ffu;
                    if (!two(g)) q_turn ^= Z::kQueryTiles - 1;
                } else {
                    wait(q_full, q_phase);
                    q_phase ^= 1;
                }
                auto queries_read = [&]() {  // when the products so far are complete
                    if constexpr (FOUR) {
                        mma_commit(tile_empty(q_tile));
                        if (two(g)) mma_commit(tile_empty(1));
                    } else {
                        mma_commit(q_empty);
                    }
                };
                if (two(g)) {
                    const uint32_t s = next_stage();
                    if (!ok) break;
                    fence_after();
                    for (int slot = 0; slot < 2; ++slot)
                        if (issuing()) scores(slot, qdesc + slot * kStep, s);
                    if (issuing()) {  // (the last keys' stage is the softmax's)
                        if (g.nt == 1)
                            queries_read();
                        else
                            mma_commit(empty_bar(s));
                    }
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
                            wait(p_half(slot), FOUR ? halves >> slot & 1 : h_phase);
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
                                outputs(slot, 32, v + kValueHalf, true);
                                if (more) {
                                    scores(slot, qdesc + slot * kStep, ks);
                                    if (slot) {
                                        if (t + 2 == g.nt)
                                            queries_read();
                                        else
                                            mma_commit(empty_bar(ks));
                                    }
                                } else {
                                    mma_commit(o_full(slot));
                                }
                                if (slot && more) mma_commit(empty_bar(vs));
                            }
                            together();
                        }
                        h_phase ^= 1;
                        halves ^= 3;
                        p_phase0 ^= 1;
                        p_phase1 ^= 1;
                    }
                } else if constexpr (FOUR) {
                    // one row tile: key tile t goes to slot t & 1, before tile t - 1's weights meet its values
                    const int nt = tiles(g);
                    uint32_t vs = stage, v_phase = stage_phase;
                    auto step = [](uint32_t &s, uint32_t &phase, uint32_t by) {
                        if ((s += by) >= S) {
                            s -= S;
                            phase ^= 1;
                        }
                    };
                    step(vs, v_phase, 1);
                    for (int t = 0; ok && t <= nt; ++t) {
                        if (t < nt) {
                            const int slot = t & 1;
                            wait(full_bar(stage), stage_phase);
                            if (!ok) break;
                            fence_after();
                            // (the slot's scores before have been read, and their weights used: those products were issued first)
                            if (issuing()) {
                                scores(slot, qdesc + q_tile * kStep, stage);
                                mma_commit(empty_bar(stage));
                                if (t == nt - 1) queries_read();
                            }
                            together();
                            step(stage, stage_phase, 2);
                        }
                        if (t > 0) {
                            const int slot = (t - 1) & 1;
                            wait(full_bar(vs), v_phase);
                            wait(p_half(slot), halves >> slot & 1);
                            if (!ok) break;
                            fence_after();
                            const uint64_t v = vdesc + vs * kStep;
                            if (issuing()) outputs(slot, 0, v, t > 2);
                            together();
                            wait(p_full(slot), slot ? p_phase1 : p_phase0);
                            if (!ok) break;
                            fence_after();
                            if (issuing()) {
                                outputs(slot, 32, v + kValueHalf, true);
                                mma_commit(empty_bar(vs));
                                if (t - 1 + 2 >= nt) mma_commit(o_full(slot));
                            }
                            together();
                            halves ^= 1u << slot;
                            if (slot)
                                p_phase1 ^= 1;
                            else
                                p_phase0 ^= 1;
                            step(vs, v_phase, 2);
                        }
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
                                scores_half(slot, s, qdesc + q_tile * kStep);
                                if (t == g.nt - 1) queries_read();
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

template <int D, bool BF16, bool FOUR = false, int P = 2>
cudaError_t launch(const AttnArgs &a, const CUtensorMap &q, const CUtensorMap &few, const CUtensorMap &k, const CUtensorMap &v, void *ws, cudaStream_t stream) {
    static std::atomic<uint64_t> prepared{0};  // devices whose kernel has been given its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev > 63 || !(prepared.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(attention_tc_kernel<D, BF16, FOUR, P>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sizes<D, FOUR, P>::kSmem);
        if (FOUR && e == cudaSuccess) {  // registers are shared out as if launched with so many
            cudaFuncAttributes f;
            e = cudaFuncGetAttributes(&f, attention_tc_kernel<D, BF16, FOUR, P>);
            if (e == cudaSuccess && f.numRegs < kLaunchRegisters) e = cudaErrorInvalidConfiguration;
        }
        if (e == cudaSuccess && dev <= 63) prepared.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
        e = launch_behind(attention_tc_kernel<D, BF16, FOUR, P>, dim3(kMaxBlocks), FOUR ? kFourbitThreads : kThreads, (size_t)Sizes<D, FOUR, P>::kSmem, stream, a, q, few, k, v, ws);
    if (e == cudaSuccess)
        e = launch_behind(attention_combine_kernel<D, typename std::conditional<BF16, uint16_t, f16_t>::type, FOUR, P>, dim3(kMaxBlocks, kCombineDims, kCombineRows), kCombineThreads, 0, stream, a, ws);
    return e;
}

}  // namespace

// `rows` of a sequence and key head on average.  Up to one row tile the kernel for such items alone is the faster one, whose code
// fits the instruction caches better (64 chunks of 32 over 4000, 32 / 8 heads x 128: 227 us, and 240 with the other; of 34: 400, 299).
template <int D, bool BF16>
static cudaError_t launch_fourbit(const AttnArgs &a, int64_t rows, void *ws, cudaStream_t stream) {
    const CUtensorMap none = {};  // (a page is copied as it lies)
    return rows <= kTile ? launch<D, BF16, true, 1>(a, none, none, none, none, ws, stream) : launch<D, BF16, true, 2>(a, none, none, none, none, ws, stream);
}

pcg_status attention_fourbit_tc(const char *who, const AttnArgs &a, pcg_dtype dtype, int64_t rows, void *ws, cudaStream_t stream) {
    cudaError_t e;
    if (a.d == 128)
        e = dtype == PCG_BF16 ? launch_fourbit<128, true>(a, rows, ws, stream) : launch_fourbit<128, false>(a, rows, ws, stream);
    else
        e = dtype == PCG_BF16 ? launch_fourbit<64, true>(a, rows, ws, stream) : launch_fourbit<64, false>(a, rows, ws, stream);
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

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
