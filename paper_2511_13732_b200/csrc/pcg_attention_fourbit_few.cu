// Attention over the cache that holds 4.5 bits a value for few rows: single tokens and short drafts, up to 32 rows of a
// key head; bfloat16 and float16 queries, head dimensions 64 and 128.
//
// Each warp works alone, on 64 keys at a time, with warp-level products whose operands are widened codes straight in registers:
//     S^T[key][row] = K[key][dim] Q^T[dim][row],   O^T[dim][row] += V^T[dim][key] P^T[key][row]
// with 16 keys, or 16 value dimensions, to 8 rows a product.  What bounds a call is then reading the cache and widening it, and
// no warp waits for another.  (64 single tokens of 32 query heads over up to 32,000, 128 dimensions: 246 us, 82 % of the
// measured copy's rate; with keys on the lanes of tensor memory and 16 columns for the four rows, where five roles hand over to
// one another for every 128 keys, 440 us.  The other path's tiles have 128 rows.  At 128 dimensions it is the faster one beyond 32;
// at 64, 32 rows are what a lane's registers hold here, and the faster there still.)
//
// What a lane holds of an operand is free where both sides agree, so lanes take what lies together in a page.  With g = lane / 4,
// i = lane % 4, and a chunk of four pages of 16 keys:
//     keys      lane (g, i) has 32 dimensions from 32 i on (64-dimensional heads: 16 from 16 i on) of token 2 b + g % 2 of page
//               g / 2, in turn b = 0 .. 7: 16 bytes of codes, and dimensions of the query to match
//     weights   S^T's block b comes out as (that key, rows 2 i and 2 i + 1), and transposed (movmatrix) as (row g, tokens 2 b and
//               2 b + 1 of page i)
//     values    lane (g, i) has dimensions g and g + 8 of 16 of all 16 tokens of page i: 8 bytes of codes each
// Pages are 32 bytes further apart in shared memory than they are long (modulo 128), which spreads them over the banks.
//
// Work is shared out as in the other kernels, but a run is a warp's: a key head's rows of one row tile are an item, parts of
// items are joined by a second kernel.
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "pcg_attention_work.cuh"
#include "pcg_fourbit.cuh"
#include "pcg_tcgen05.cuh"

namespace pcg {

namespace {

constexpr int kChunk = 64;      // keys of a warp's turn
constexpr float kSlack = 8.f;   // the reference may lag the maximum by a factor 2^8 before sums are scaled
constexpr float kLift = 7.f;    // float16 weights are kept 2^7 higher, out of the range where they lose bits
// (joining costs little: one stream of 5 tokens over 3001 takes 21.2 us with runs of one chunk, 21.5 of two, 25.4 of three)
constexpr int kFewItemUnits = 1, kFewLeast = 1;

template <int D, int NT>
struct Few {
    static constexpr int kWarps = NT <= 2 ? 12 : 7;
    static constexpr int kRuns = kMaxBlocks * kWarps;
    static constexpr int kRows = 8 * NT;
    static constexpr int kTurns = NT == 1 ? 1 : 2;  // a chunk's keys are taken in (registers: two halves)
    static constexpr int kPitch = (page_bytes(D) + 127) / 128 * 128 + 32;  // of a page in shared memory
    static constexpr int kStage = 4 * kPitch;
    static constexpr int kStages = 225 * 1024 / (kWarps * kStage) < 4 ? 225 * 1024 / (kWarps * kStage) : 4;
    static constexpr int kSmem = kWarps * kStages * kStage > kAttnMaxB * 12 ? kWarps * kStages * kStage : kAttnMaxB * 12;
    static_assert(kStages >= 2, "a stage to read, one to fill");
};
// At the head of the workspace; the parts of items lie behind it: [run][2: one that does not begin its item, one that does]
// [rows][D] sums, then references, then sums of weights.
template <int RUNS>
struct FewHead {
    Run run[RUNS + 1];
    int32_t failed[kMaxBlocks];
};
template <int D, int NT>
__device__ __forceinline__ float *few_part(void *ws, int run, int which) {
    constexpr size_t kHead = (sizeof(FewHead<Few<D, NT>::kRuns>) + 255) / 256 * 256;
    return reinterpret_cast<float *>((char *)ws + kHead) + ((size_t)run * 2 + which) * Few<D, NT>::kRows * (D + 2);
}
template <int D, int NT>
constexpr size_t few_bytes() {
    return (sizeof(FewHead<Few<D, NT>::kRuns>) + 255) / 256 * 256 + (size_t)Few<D, NT>::kRuns * 2 * Few<D, NT>::kRows * (D + 2) * 4;
}

// c[16][8] += a[16][16] b[16][8]
__device__ __forceinline__ void product(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turned(uint32_t x) {  // a warp's 8 x 8 matrix of 16-bit values
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t r;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 r;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(at) : "memory");
    return r;
}

template <typename T>
__device__ __forceinline__ uint32_t round_pair(float lo, float hi) {
    return std::is_same<T, uint16_t>::value ? pack2<true>(lo, hi) : pack2<false>(lo, hi);
}

template <int D, int NT, typename T>
__global__ void __launch_bounds__(32 * Few<D, NT>::kWarps, 1)
    attention_fourbit_few_kernel(const __grid_constant__ AttnArgs a, void *ws) {
    using Z = Few<D, NT>;
    constexpr int W = Z::kWarps, S = Z::kStages, kPage = page_bytes(D), QR = D / 8;  // QR: a lane's registers of 8 queries
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ int64_t warp_units[W], warp_items[W];
    __shared__ Run run[2 * W];
    __shared__ __align__(8) uint64_t bars[W * S];
    __shared__ int failed_flag;
    volatile int *failed = &failed_flag;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lg = lane >> 2, li = lane & 3;
    const uint32_t ring = smem_u32(smem_raw) + warp * S * Z::kStage, bar0 = smem_u32(bars) + 8u * warp * S;
    if (tid == 0) {
        for (int i = 0; i < W * S; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(bars) + 8u * i));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed_flag = 0;
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int G = a.q_heads / a.kv_heads, TQ = Z::kRows / G;
    cut_work<kFewItemUnits, kFewLeast, 1, W>(a, TQ, reinterpret_cast<int64_t *>(smem_raw), warp_units, warp_items, run);
    FewHead<Z::kRuns> *head = reinterpret_cast<FewHead<Z::kRuns> *>(ws);
    // (runs are dealt out over the blocks first: the few runs of a small call have an SM each)
    if (tid < W) head->run[tid * kMaxBlocks + blockIdx.x] = run[2 * tid];
    if (tid == 0 && blockIdx.x == kMaxBlocks - 1) head->run[Z::kRuns] = run[2 * W - 1];

    Walk walk, ahead;  // where the products are, and the copies
    walk.start(a, run[2 * warp], run[2 * warp + 1]);
    ahead = walk;
    Segment g, f;
    auto last_key = [](const Segment &g) { return min(g.len, (g.t0 + g.nt) * kChunk); };
    // Copies of one chunk ahead: a lane a page.  The next chunk's blocks are looked up before this one's are needed.
    bool more = ahead.next<1>(a, TQ, f);
    int at = 0, stage_in = 0;
    uint32_t asked = 0;
    auto block_of = [&]() -> int32_t {  // of the lane's page: -1 none there, -2 zeros
        const int p = (f.t0 + at) * kChunk + lane * 16;
        if (!more || lane >= 4 || p >= last_key(f)) return -1;
        const int32_t block = a.block_table[(int64_t)f.b * a.max_blocks + (p >> a.bs_shift)];
        return block < 0 || block >= a.n_blocks ? -2 : block;
    };
    int32_t block = block_of();
    auto fetch = [&]() {
        if (!more) return;
        const int p = (f.t0 + at) * kChunk + (lane & 3) * 16;
        const int64_t in = (p & ((1 << a.bs_shift) - 1)) >> 4;
        const uint8_t *src = (const uint8_t *)a.k + ((((int64_t)max(block, 0) * a.kv_heads + f.h) << (a.bs_shift - 4)) + in) * kPage;
        const uint32_t dst = ring + stage_in * Z::kStage, bar = bar0 + 8u * stage_in;
        if (__any_sync(0xffffffffu, block == -2)) {
            if (block == -2)
                for (int i = 0; i < kPage; i += 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + lane * Z::kPitch + i), "r"(0u) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        const uint32_t there = __ballot_sync(0xffffffffu, block >= 0);
        if (elect_one()) bar_expect(bar, __popc(there) * kPage);
        __syncwarp();
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
            const uint64_t from = __shfl_sync(0xffffffffu, (unsigned long long)(uintptr_t)src, c);
            if ((there >> c & 1) && elect_one())
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + c * Z::kPitch), "l"(from),
                             "r"(kPage), "r"(bar)
                             : "memory");
            __syncwarp();
        }
        ++asked;
        if (++stage_in == S) stage_in = 0;
        if (++at == f.nt) {
            at = 0;
            more = ahead.next<1>(a, TQ, f);
        }
        block = block_of();
    };
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) fetch();

    uint32_t stage = 0, phase = 0;
    bool ok = true;
    while (ok && walk.next<1>(a, TQ, g)) {
        const int tokens = min(g.n - g.pair * TQ, TQ), rows = tokens * G, k_end = last_key(g);
        const int seen0 = g.len - g.n + g.pair * TQ + 1;  // keys that the first token sees
        // ---- queries: row 8 j + g, the lane's dimensions
        uint32_t q[NT][QR];
        float by_q[NT][2], ref[NT][2];  // of rows 2 i and 2 i + 1: what products are multiplied by, references (0 until there is one)
        int lim[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int r = 8 * j + lg, tok = r / G;
            const T *src = (const T *)a.q + ((int64_t)g.begin + g.pair * TQ + tok) * a.q_stride + ((int64_t)g.h * G + (r - tok * G)) * D + li * (D / 4);
            float by = a.scale_log2;
            uint4 w[D / 32];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) w[c] = r < rows ? reinterpret_cast<const uint4 *>(src)[c] : make_uint4(0u, 0u, 0u, 0u);
            if constexpr (std::is_same<T, uint16_t>::value) by *= narrow_row<4>(w);
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                q[j][c * 4] = w[c].x;
                q[j][c * 4 + 1] = w[c].y;
                q[j][c * 4 + 2] = w[c].z;
                q[j][c * 4 + 3] = w[c].w;
            }
            by = fminf(fmaxf(by, 1.17549435e-38f), 3.40282347e38f);  // (never 0: 0 times a masked score would be NaN)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                by_q[j][e] = __shfl_sync(0xffffffffu, by, (2 * li + e) * 4);
                const int row = 8 * j + 2 * li + e;
                lim[j][e] = row < rows ? min(seen0 + row / G, k_end) : 0x7fffffff;  // (padding's scores are 0, and of no matter)
                ref[j][e] = 0.f;
            }
        }
        float o[D / 16][NT][4], l[NT][2];
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int j = 0; j < NT; ++j) o[c][j][0] = o[c][j][1] = o[c][j][2] = o[c][j][3] = 0.f;
#pragma unroll
        for (int j = 0; j < NT; ++j) l[j][0] = l[j][1] = 0.f;
        const int least = min(seen0, k_end);  // keys that every row sees

#pragma unroll 1
        for (int t = 0; t < g.nt; ++t) {
            const int k0 = (g.t0 + t) * kChunk;
            ok = __all_sync(0xffffffffu, bar_wait_hot(bar0 + 8u * stage, phase, failed));
            if (!ok) break;
            const uint32_t page0 = ring + stage * Z::kStage;
            fetch();  // into the stage that the last turn has read
            const uint32_t key = page0 + (lg >> 1) * Z::kPitch, page = page0 + li * Z::kPitch;
            constexpr int M = 4 / Z::kTurns;  // products of 16 keys a turn; twice as many blocks, from 2 M h on
#pragma unroll 1
            for (int h = 0; h < Z::kTurns; ++h) {
                // ---- scores: products of 16 keys, two blocks
                float s[M][NT][4];
#pragma unroll
                for (int c = 0; c < M; ++c) {
                    uint32_t w[2][D / 32], by[2][2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int tok = 4 * M * h + 4 * c + 2 * e + (lg & 1);
                        if constexpr (D == 128) {
                            const uint4 x = lds128(key + li * 256 + tok * 16);
                            w[e][0] = x.x, w[e][1] = x.y, w[e][2] = x.z, w[e][3] = x.w;
                            uint16_t two;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(two) : "r"(key + key_scales_at(D) + tok * 8 + li * 2) : "memory");
                            uint32_t f2[2];
                            widen_scales(two, f2);
                            by[e][0] = __byte_perm(f2[0], f2[0], 0x1010);
                            by[e][1] = __byte_perm(f2[0], f2[0], 0x3232);
                        } else {
                            const uint2 x = lds64(key + (li >> 1) * 256 + tok * 16 + (li & 1) * 8);
                            w[e][0] = x.x, w[e][1] = x.y;
                            uint16_t one;
                            asm volatile("{\n\t.reg .u8 t;\n\tld.shared.u8 t, [%1];\n\tcvt.u16.u8 %0, t;\n\t}" : "=h"(one) : "r"(key + key_scales_at(D) + tok * 4 + li) : "memory");
                            uint32_t f2[2];
                            widen_scales(one, f2);
                            by[e][0] = by[e][1] = __byte_perm(f2[0], f2[0], 0x1010);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < NT; ++j) s[c][j][0] = s[c][j][1] = s[c][j][2] = s[c][j][3] = 0.f;
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {  // a word: eight dimensions, two products
                        uint32_t v0[4], v1[4];
                        widen_codes(w[0][x], v0);
                        widen_codes(w[1][x], v1);
                        const int half = D == 128 ? x >> 1 : 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v0[e] = mul_f16x2(v0[e], by[0][half]);
                            v1[e] = mul_f16x2(v1[e], by[1][half]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; e += 2)
#pragma unroll
                            for (int j = 0; j < NT; ++j) product(s[c][j], v0[e], v1[e], v0[e + 1], v1[e + 1], q[j][x * 4 + e], q[j][x * 4 + e + 1]);
                    }
                }
                if (k0 + kChunk > least) {  // keys that a row does not see
                    const int k = k0 + (lg >> 1) * 16 + (lg & 1) + 4 * M * h;
#pragma unroll
                    for (int c = 0; c < M; ++c)
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (k + 4 * c + (e & 2) >= lim[j][e & 1]) s[c][j][e] = kNegInf;
                }
                // ---- weights
                float most[NT][2], top = kNegInf;  // the lane's largest; how far a score is above its row's reference
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        most[j][e] = kNegInf;
#pragma unroll
                        for (int c = 0; c < M; ++c) most[j][e] = fmaxf(most[j][e], fmaxf(s[c][j][e], s[c][j][e + 2]));
                        top = fmaxf(top, fmaf(most[j][e], by_q[j][e], -ref[j][e]));
                    }
                // (the first half's references are its own maxima, whatever they are)
                const bool first = t == 0 && h == 0;
                if (__any_sync(0xffffffffu, first || top > kSlack)) {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
#pragma unroll
                            for (int w = 4; w < 32; w <<= 1) most[j][e] = fmaxf(most[j][e], __shfl_xor_sync(0xffffffffu, most[j][e], w));
                            most[j][e] *= by_q[j][e];
                            const bool up = first ? most[j][e] > kNegInf : most[j][e] > ref[j][e] + kSlack;
                            const float by = up ? ex2(ref[j][e] - most[j][e]) : 1.f;
                            if (up) ref[j][e] = most[j][e];
                            l[j][e] *= by;
#pragma unroll
                            for (int c = 0; c < D / 16; ++c) {
                                o[c][j][e] *= by;
                                o[c][j][e + 2] *= by;
                            }
                        }
                }
                // Weights are rounded to float16, the type of the other operand: the products take two of one 16-bit type, and of
                // those it has the most bits.  That is off by 2^-12 of a weight at most, which an output in float16 shows (2.8e-4
                // in 2-norm where its own rounding gives 2.1e-4) and one in bfloat16 does not (1.7e-3 either way).  Their sum is
                // float32, of the weights before the rounding.
                uint32_t p[2 * M][NT];  // of block 2 M h + b: (row g, tokens 2 b and 2 b + 1 behind 4 M h of page i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const float r0 = kLift - ref[j][0], r1 = kLift - ref[j][1];
#pragma unroll
                    for (int c = 0; c < M; ++c)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float x0 = ex2(fmaf(s[c][j][2 * e], by_q[j][0], r0)), x1 = ex2(fmaf(s[c][j][2 * e + 1], by_q[j][1], r1));
                            l[j][0] += x0;
                            l[j][1] += x1;
                            p[2 * c + e][j] = turned(pack2<false>(x0, x1));
                        }
                }
                // ---- outputs: 16 dimensions at a time.  Scales of tokens behind the part's last key, which may be anything, are 0.
                const int left = k_end - k0 - li * 16 - 4 * M * h;  // tokens of the lane's
                uint32_t keep[M];
#pragma unroll
                for (int w = 0; w < M; ++w) {
                    const int n = left - 4 * w;
                    keep[w] = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                }
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const uint32_t scales = page + value_scales_at(D) + c * 16 + 4 * M * h, codes = page + value_codes_at(D) + (c * 16 + lg) * 8 + 2 * M * h;
                    uint32_t w[M], c0[M / 2], c1[M / 2];
                    if constexpr (M == 4) {
                        const uint4 x = lds128(scales);
                        const uint2 y0 = lds64(codes), y1 = lds64(codes + 64);
                        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
                        c0[0] = y0.x, c0[1] = y0.y, c1[0] = y1.x, c1[1] = y1.y;
                    } else {
                        const uint2 x = lds64(scales);
                        w[0] = x.x, w[1] = x.y;
                        c0[0] = lds32(codes), c1[0] = lds32(codes + 64);
                    }
#pragma unroll
                    for (int y = 0; y < M / 2; ++y) {
                        uint32_t by[4], v0[4], v1[4];
                        widen_scales(w[2 * y] & keep[2 * y], reinterpret_cast<uint32_t(&)[2]>(by[0]));
                        widen_scales(w[2 * y + 1] & keep[2 * y + 1], reinterpret_cast<uint32_t(&)[2]>(by[2]));
                        widen_codes(c0[y], v0);
                        widen_codes(c1[y], v1);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v0[e] = mul_f16x2(v0[e], by[e]);
                            v1[e] = mul_f16x2(v1[e], by[e]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; e += 2)
#pragma unroll
                            for (int j = 0; j < NT; ++j) product(o[c][j], v0[e], v1[e], v0[e + 1], v1[e + 1], p[4 * y + e][j], p[4 * y + e + 1][j]);
                    }
                }
            }
            __syncwarp();  // the stage has been read
            if (++stage == S) {
                stage = 0;
                phase ^= 1;
            }
        }
        if (!ok) break;
        // ---- end of the part
        float *part = few_part<D, NT>(ws, warp * kMaxBlocks + blockIdx.x, g.t0 == 0 ? 1 : 0);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float inv[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) l[j][e] += __shfl_xor_sync(0xffffffffu, l[j][e], w);
                inv[e] = a.v_scale / l[j][e];  // a row that sees scores of -inf alone is 0 / 0 = NaN
                const int row = 8 * j + 2 * li + e;
                if (!g.whole && lg == 0 && row < rows) {
                    part[Z::kRows * D + row] = l[j][e] == 0.f ? kNegInf : ref[j][e];  // (nothing seen: no reference)
                    part[Z::kRows * (D + 1) + row] = l[j][e];
                }
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                if (g.whole) {
                    // two rows of a dimension a lane, turned: two dimensions of a row
                    const int r = 8 * j + lg, tok = r / G;
                    const bool empty = seen0 + tok <= 0;  // a row that sees no key is 0
                    T *to = (T *)a.out + (((int64_t)g.begin + g.pair * TQ + tok) * a.q_heads + (int64_t)g.h * G + (r - tok * G)) * D + c * 16 + 2 * li;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t w = turned(round_pair<T>(o[c][j][2 * h] * inv[0], o[c][j][2 * h + 1] * inv[1]));
                        if (r < rows) *reinterpret_cast<uint32_t *>(to + 8 * h) = empty ? 0u : w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = 8 * j + 2 * li + (e & 1);
                        if (row < rows) part[(size_t)row * D + c * 16 + lg + (e & 2) * 4] = o[c][j][e];
                    }
                }
            }
        }
    }
    if (!ok) {  // giving up: copies already asked for may still be landing
        for (uint32_t back = 1; back <= S && back <= asked; ++back) bar_drain(bar0 + 8u * ((asked - back) % S), ((asked - back) / S) & 1);
    }
    __syncthreads();
    if (tid == 0) head->failed[blockIdx.x] = failed_flag;
}

// Joins the items that several runs had a part in.  Every block lists them for itself (the heads of all runs, out of L2); a warp
// takes a row of one, a lane D / 32 dimensions; rows lie over all SMs first.  What bounds it is the latency of three rounds of
// loads: heads, references, sums, of eight parts at a time.  (One stream of 5 tokens over 3001, 47 parts an item: 6 us of 21;
// rows packed into few blocks and sums behind their references 13 of 28.  A block for each run, most of which have nothing to
// join, took 14 us to come and go.)
constexpr int kJoinThreads = 1024, kAtOnce = 8;  // parts whose sums are asked for together

template <int D, int NT, typename T>
__global__ void __launch_bounds__(kJoinThreads) attention_fourbit_few_join_kernel(const __grid_constant__ AttnArgs a, void *ws) {
    using Z = Few<D, NT>;
    constexpr int kPer = (Z::kRuns + kJoinThreads - 1) / kJoinThreads, N = D / 32;
    __shared__ int64_t first_of[Z::kRuns + 1];
    __shared__ int16_t begins[Z::kRuns];  // runs that begin an item that others go on with
    __shared__ int warp_count[kJoinThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const FewHead<Z::kRuns> *head = reinterpret_cast<const FewHead<Z::kRuns> *>(ws);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lo = min(Z::kRuns, tid * kPer), hi = min(Z::kRuns, lo + kPer);
    int64_t next_first[kPer];
    int next_tile[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const Run *r = &head->run[min(lo + i + 1, Z::kRuns)];
        next_first[i] = r->first;
        next_tile[i] = r->tile;
    }
    const int64_t all = head->run[Z::kRuns].first;
    const bool bad = tid < kMaxBlocks && head->failed[tid];
    uint32_t mine = 0;  // bit c - lo: run c is one
    int64_t begun = head->run[lo].first;
    first_of[lo] = begun;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int c = lo + i;
        if (c >= hi) break;
        const int64_t next = next_first[i];
        const int tile = next_tile[i];
        if (next < all && tile != 0 && next - tile >= begun) mine |= 1u << i;
        first_of[c + 1] = begun = next;
    }
    if (__syncthreads_or(bad)) {  // no row may pass for a result
        const uint32_t nan2 = 0x7fff7fffu;  // NaN in both types
        const int64_t vecs = (int64_t)a.rows * a.q_heads * (D * (int)sizeof(T) / 16);
        for (int64_t i = (int64_t)blockIdx.x * kJoinThreads + tid; i < vecs; i += (int64_t)gridDim.x * kJoinThreads)
            reinterpret_cast<uint4 *>(a.out)[i] = make_uint4(nan2, nan2, nan2, nan2);
        return;
    }
    int count = __popc(mine), before = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += up;
    }
    if (lane == 31) warp_count[warp] = before;
    __syncthreads();
    int items = 0;
    before -= count;
    for (int w = 0; w < kJoinThreads / 32; ++w) {
        if (w < warp) before += warp_count[w];
        items += warp_count[w];
    }
    for (; mine; mine &= mine - 1) begins[before++] = (int16_t)(lo + __ffs(mine) - 1);
    __syncthreads();
    const int G = a.q_heads / a.kv_heads, TQ = Z::kRows / G;
    for (int w = warp * gridDim.x + blockIdx.x; w < items * Z::kRows; w += gridDim.x * (kJoinThreads / 32)) {
        const int c = begins[w / Z::kRows], r = w % Z::kRows;
        const Run next = head->run[c + 1];
        int begin, n, len;
        attn_sequence(a, next.b, begin, n, len);
        if (r >= min(n - next.pair * TQ, TQ) * G) continue;
        const int64_t end = next.first - next.tile + tiles_of<1>(n, len, TQ, next.pair);
        int last = c + 1, above = Z::kRuns;  // the last run that begins before the item's end
        while (last + 1 < above) {
            const int mid = (last + above) >> 1;
            if (first_of[mid] < end)
                last = mid;
            else
                above = mid;
        }
        // the first part lies among its run's parts that begin an item, the others among those that do not
        const float *first = few_part<D, NT>(ws, c, 1), *rest = few_part<D, NT>(ws, c + 1, 0);
        constexpr int64_t kStride = 2 * (int64_t)Z::kRows * (D + 2), kM = (int64_t)Z::kRows * D, kL = kM + Z::kRows;
        const int parts = last - c, dim = lane * N;
        const float m0 = first[kM + r];
        float m = m0;
        for (int k = lane; k < parts; k += 32) m = fmaxf(m, rest[k * kStride + kM + r]);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
        auto factor = [&](float mk) { return mk == kNegInf ? 0.f : mk == m ? 1.f : ex2(mk - m); };
        const float f0 = factor(m0);
        float l = lane == 0 ? first[kL + r] * f0 : 0.f, o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = first[(int64_t)r * D + dim + i] * f0;
#pragma unroll 1
        for (int k0 = 0; k0 < parts; k0 += 32) {  // a part's factor and sum of weights a lane
            const float *mine = rest + (k0 + lane) * kStride + r;
            const bool there = k0 + lane < parts;
            const float f = there ? factor(mine[kM]) : 0.f;
            if (there) l += mine[kL] * f;
#pragma unroll 1
            for (int k = k0; k < min(k0 + 32, parts); k += kAtOnce) {
                float2 x[kAtOnce][N / 2];
#pragma unroll
                for (int e = 0; e < kAtOnce; ++e) {
                    const float2 *v = reinterpret_cast<const float2 *>(rest + (k + e) * kStride + (int64_t)r * D + dim);
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) x[e][i] = k + e < parts ? v[i] : make_float2(0.f, 0.f);
                }
#pragma unroll
                for (int e = 0; e < kAtOnce; ++e) {
                    const float fe = __shfl_sync(0xffffffffu, f, k - k0 + e);
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) {
                        o[2 * i] += x[e][i].x * fe;
                        o[2 * i + 1] += x[e][i].y * fe;
                    }
                }
            }
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        const int tok = r / G, t_row = next.pair * TQ + tok;
        const bool empty = len - n + t_row + 1 <= 0;
        uint32_t *to = reinterpret_cast<uint32_t *>((T *)a.out + (((int64_t)begin + t_row) * a.q_heads + (int64_t)next.h * G + (r - tok * G)) * D + dim);
        const float inv = a.v_scale / l;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) to[i] = empty ? 0u : round_pair<T>(o[2 * i] * inv, o[2 * i + 1] * inv);
    }
}

template <int D, int NT, typename T>
cudaError_t launch(const AttnArgs &a, void *ws, cudaStream_t stream) {
    using Z = Few<D, NT>;
    static_assert(few_bytes<D, NT>() <= 148ull * 2 * 256 * (D + 2) * 4 + 4096, "the workspace");
    static std::atomic<uint64_t> prepared{0};  // devices whose kernel has been given its shared memory
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev > 63 || !(prepared.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(attention_fourbit_few_kernel<D, NT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Z::kSmem);
        if (e == cudaSuccess && dev <= 63) prepared.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
        e = launch_behind(attention_fourbit_few_kernel<D, NT, T>, dim3(kMaxBlocks), 32 * Z::kWarps, (size_t)Z::kSmem, stream, a, ws);
    if (e == cudaSuccess)
        e = launch_behind(attention_fourbit_few_join_kernel<D, NT, T>, dim3(kMaxBlocks), kJoinThreads, 0, stream, a, ws);
    return e;
}

template <int D, typename T>
cudaError_t dispatch(const AttnArgs &a, int tile_rows, void *ws, cudaStream_t stream) {
    if (tile_rows <= 8) return launch<D, 1, T>(a, ws, stream);
    if (tile_rows <= 16) return launch<D, 2, T>(a, ws, stream);
    if constexpr (D == 64)
        if (tile_rows > 24) return launch<D, 4, T>(a, ws, stream);
    return launch<D, 3, T>(a, ws, stream);
}

}  // namespace

pcg_status attention_fourbit_few(const char *who, const AttnArgs &a, pcg_dtype dtype, int tile_rows, void *ws, cudaStream_t stream) {
    cudaError_t e;
    if (a.d == 128)
        e = dtype == PCG_BF16 ? dispatch<128, uint16_t>(a, tile_rows, ws, stream) : dispatch<128, f16_t>(a, tile_rows, ws, stream);
    else
        e = dtype == PCG_BF16 ? dispatch<64, uint16_t>(a, tile_rows, ws, stream) : dispatch<64, f16_t>(a, tile_rows, ws, stream);
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

}  // namespace pcg
