// Attention in float32 on the FMA pipes, head dimensions 64 and 128: the work is shared out as for the tensor cores
// (pcg_attention_work.cuh), a block's run is gone through 64 or 32 rows by 64 keys at a time.
//
// Thread (ty, tx) of 16 x 16 has rows R ty .. R ty + R - 1, R = 4 or 2: their scores with keys tx, tx + 16, tx + 32, tx + 48, and their
// outputs in dimensions 4 tx .. (and 64 + 4 tx ..).  Operands come out of shared memory as 16-byte vectors, sixteen products
// for two of them; keys and values of the next 64 keys arrive (cp.async) while these are worked on.  Warps whose rows are all
// padding, as most are for a drafted chunk's few rows, skip the arithmetic.
// What bounds it: the FMA pipes for chunks of prompts; for few rows the latency of a run's steps (16 chunks of 9 rows over up
// to 700 tokens, 12 / 4 heads x 64: 29 us for 14 MB; a block per row and head took 109).  Prompts: 2048 tokens, 12 / 4 heads x 64,
// 355 us (18 TFLOP/s), 32 / 8 x 128, 1201 us (29 TFLOP/s).
#include <atomic>
#include <cstddef>
#include <type_traits>

#include "pcg_attention_work.cuh"

namespace pcg {

constexpr int kF32Threads = 256, kF32Rows = 64, kF32Keys = 64;

template <int D>
struct F32Shared {
    int64_t sums[2][kF32Threads / 32];  // the cut's
    Run run[2];
    alignas(16) float q[kF32Rows][D + 4];
    float k[2][kF32Keys][D + 4];
    float v[2][kF32Keys][D + 4];
    float p[kF32Rows][kF32Keys + 4];
};

__device__ __forceinline__ void copy16(void *to, const void *from, bool there) {  // zeros where nothing is there
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0)
                 : "memory");
}

template <int D>
__global__ void __launch_bounds__(kF32Threads, 1) attention_f32_kernel(const __grid_constant__ AttnArgs a, void *ws) {
    constexpr int V = D / 4, N = D / 64;  // vectors of a row; vectors of a thread's outputs in a row
    extern __shared__ __align__(16) unsigned char smem_raw[];
    F32Shared<D> &sh = *reinterpret_cast<F32Shared<D> *>(smem_raw);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int G = a.q_heads / a.kv_heads, TQ = kTile / G;
    // the cut's scratch, 12 bytes a sequence, lies over the tiles
    cut_work(a, TQ, reinterpret_cast<int64_t *>(sh.q), sh.sums[0], sh.sums[1], sh.run);
    WorkspaceHead *head = reinterpret_cast<WorkspaceHead *>(ws);
    if (tid == 0) {
        head->run[blockIdx.x] = sh.run[0];
        head->failed[blockIdx.x] = 0;
        if (blockIdx.x == kMaxBlocks - 1) head->run[kMaxBlocks] = sh.run[1];
    }
    Walk walk;
    walk.start(a, sh.run[0], sh.run[1]);
    __syncthreads();
    Segment g;
    while (walk.next(a, TQ, g)) {
        const int keys = g.two ? kTile : kHalf;
        const int k_begin = g.t0 * keys, k_end = min((g.t0 + g.nt) * keys, g.len);
        const int tokens = min(g.n - g.pair * 2 * TQ, 2 * TQ);
        float *part = part_base(ws, blockIdx.x, g.t0 == 0 ? 1 : 0, D);
        // Row r of tile r / 128 has token (r / 128) TQ + (r % 128) / G.  16 * R rows from r0 on, R of them a thread.
        auto work = [&](auto rows_each, int r0) {
            constexpr int R = decltype(rows_each)::value, kRows = 16 * R;
            auto token_of = [&](int r) {  // of the row in its sequence, or -1
                const int in = r & (kTile - 1), tok = (r / kTile) * TQ + in / G;
                return in / G >= TQ || tok >= tokens ? -1 : g.pair * 2 * TQ + tok;
            };
            int lim[R];
            bool any = false;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int t = token_of(r0 + R * ty + i);
                lim[i] = t < 0 ? 0 : g.len - g.n + t + 1;
                any = any || t >= 0;
            }
            any = __any_sync(0xffffffffu, any);
            // what the last of these rows sees
            int last = token_of(r0 + kRows - 1);
            if (last < 0) last = r0 < kTile && tokens > TQ ? g.pair * 2 * TQ + TQ - 1 : g.pair * 2 * TQ + tokens - 1;
            const int k_stop = min(k_end, g.len - g.n + last + 1);
            for (int i = tid; i < kRows * V; i += kF32Threads) {
                const int r = i / V, c = i % V, t = token_of(r0 + r);
                const float *from = (const float *)a.q + ((int64_t)g.begin + max(t, 0)) * a.q_stride +
                                    (int64_t)(g.h * G + ((r0 + r) & (kTile - 1)) % G) * D + c * 4;
                copy16(&sh.q[r][c * 4], from, t >= 0);
            }
            // Thread t copies vector t % V of rows t / V, t / V + 256 / V, ...; the blocks of those rows are looked up one tile
            // ahead of the copies.
            constexpr int kCopies = kF32Keys * V / kF32Threads;
            int32_t block[kCopies];
            auto look_up = [&](int k0) {
#pragma unroll
                for (int j = 0; j < kCopies; ++j) {
                    const int pos = k0 + tid / V + j * (kF32Threads / V);
                    block[j] = a.kv_len && pos < k_stop ? a.block_table[(int64_t)g.b * a.max_blocks + (pos >> a.bs_shift)] : 0;
                }
            };
            auto fetch = [&](int k0, int buf) {
#pragma unroll
                for (int j = 0; j < kCopies; ++j) {
                    const int r = tid / V + j * (kF32Threads / V), c = tid % V, pos = k0 + r;
                    bool there = pos < k_stop;
                    int64_t ko = 0, vo = 0;
                    if (a.kv_len) {
                        there = there && block[j] >= 0 && block[j] < a.n_blocks;
                        if (there) ko = vo = ((((int64_t)block[j] * a.kv_heads + g.h) << a.bs_shift) + (pos & ((1 << a.bs_shift) - 1))) * D;
                    } else if (there) {
                        ko = ((int64_t)g.begin + pos) * a.k_stride + (int64_t)g.h * D;
                        vo = ((int64_t)g.begin + pos) * a.v_stride + (int64_t)g.h * D;
                    }
                    copy16(&sh.k[buf][r][c * 4], (const float *)a.k + ko + c * 4, there);
                    copy16(&sh.v[buf][r][c * 4], (const float *)a.v + vo + c * 4, there);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                look_up(k0 + kF32Keys);
            };
            look_up(k_begin);
            float m[R], l[R], o[R][4 * N];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                m[i] = kNegInf;
                l[i] = 0.f;
#pragma unroll
                for (int j = 0; j < 4 * N; ++j) o[i][j] = 0.f;
            }
            fetch(k_begin, 0);  // (with the queries, in one group)
            int buf = 0;
            for (int k0 = k_begin; k0 < k_stop; k0 += kF32Keys, buf ^= 1) {
                fetch(k0 + kF32Keys, buf ^ 1);  // nothing behind the last
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncthreads();
                if (any) {
                    float s[R][4];
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
                    for (int c = 0; c < D; c += 4) {
                        float4 x[R], y[4];
#pragma unroll
                        for (int i = 0; i < R; ++i) x[i] = *reinterpret_cast<const float4 *>(&sh.q[R * ty + i][c]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4 *>(&sh.k[buf][tx + 16 * j][c]);
#pragma unroll
                        for (int i = 0; i < R; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                s[i][j] = fmaf(x[i].x, y[j].x, s[i][j]);
                                s[i][j] = fmaf(x[i].y, y[j].y, s[i][j]);
                                s[i][j] = fmaf(x[i].z, y[j].z, s[i][j]);
                                s[i][j] = fmaf(x[i].w, y[j].w, s[i][j]);
                            }
                    }
#pragma unroll
                    for (int i = 0; i < R; ++i) {
                        float top = kNegInf;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            s[i][j] = k0 + tx + 16 * j < lim[i] ? s[i][j] * a.scale_log2 : kNegInf;
                            top = fmaxf(top, s[i][j]);
                        }
#pragma unroll
                        for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                        if (top > m[i]) {
                            const float f = exp2f(m[i] - top);  // 0 the first time
                            l[i] *= f;
#pragma unroll
                            for (int j = 0; j < 4 * N; ++j) o[i][j] *= f;
                            m[i] = top;
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            // masked places and scores of -inf weigh 0, whatever the reference is
                            const float w = s[i][j] == kNegInf ? 0.f : exp2f(s[i][j] - m[i]);
                            l[i] += w;
                            sh.p[R * ty + i][tx + 16 * j] = w;
                        }
                    }
                    __syncwarp();  // a row's weights come from 16 lanes of this warp
#pragma unroll 2
                    for (int c = 0; c < kF32Keys; c += 4) {
                        float4 w[R];
#pragma unroll
                        for (int i = 0; i < R; ++i) w[i] = *reinterpret_cast<const float4 *>(&sh.p[R * ty + i][c]);
#pragma unroll
                        for (int n = 0; n < N; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float4 y = *reinterpret_cast<const float4 *>(&sh.v[buf][c + e][64 * n + 4 * tx]);
#pragma unroll
                                for (int i = 0; i < R; ++i) {
                                    const float x = e == 0 ? w[i].x : e == 1 ? w[i].y : e == 2 ? w[i].z : w[i].w;
                                    o[i][4 * n] = fmaf(x, y.x, o[i][4 * n]);
                                    o[i][4 * n + 1] = fmaf(x, y.y, o[i][4 * n + 1]);
                                    o[i][4 * n + 2] = fmaf(x, y.z, o[i][4 * n + 2]);
                                    o[i][4 * n + 3] = fmaf(x, y.w, o[i][4 * n + 3]);
                                }
                            }
                    }
                }
                __syncthreads();  // the buffers are read
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
            for (int i = 0; i < R; ++i) {
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
                const int r = r0 + R * ty + i, t = token_of(r);
                if (t < 0) continue;
                if (g.whole) {
                    const float inv = 1.f / l[i];  // 0 / 0 where every score was -inf
                    float *out = (float *)a.out + (((int64_t)g.begin + t) * a.q_heads + g.h * G + (r & (kTile - 1)) % G) * D + 4 * tx;
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        *reinterpret_cast<float4 *>(out + 64 * n) =
                            lim[i] <= 0 ? make_float4(0.f, 0.f, 0.f, 0.f)
                                        : make_float4(o[i][4 * n] * inv, o[i][4 * n + 1] * inv, o[i][4 * n + 2] * inv, o[i][4 * n + 3] * inv);
                } else {
#pragma unroll
                    for (int j = 0; j < 4 * N; ++j) part[(size_t)((j >> 2) * 64 + 4 * tx + (j & 3)) * kPartRows + r] = o[i][j];
                    if (tx == 0) {
                        part[(size_t)D * kPartRows + r] = m[i];
                        part[(size_t)(D + 1) * kPartRows + r] = l[i];
                    }
                }
            }
            __syncthreads();  // the queries are read
                };
        // 64 rows at a time, and 32 where no more are left: with four rows a thread, more than half of the warps would have
        // nothing to do (four, then two rows a thread: 15 rows over 300 tokens 20.9 -> 18.1 us, 16 x 68 over 1500 354 -> 322;
        // 16 x 27 over up to 700, where each way most warps work or wait on one another, 28.4 -> 29.3)
        for (int tile = 0; tile < (g.two ? 2 : 1); ++tile) {
            const int rows = min(tokens - tile * TQ, TQ) * G;
            for (int r = 0; r < rows;) {
                if (rows - r <= 32) {
                    work(std::integral_constant<int, 2>{}, tile * kTile + r);
                    r += 32;
                } else {
                    work(std::integral_constant<int, 4>{}, tile * kTile + r);
                    r += 64;
                }
            }
        }
    }
}

namespace {

template <int D>
cudaError_t launch(const AttnArgs &a, void *ws, cudaStream_t stream) {
    // the tiles, or the cut's scratch where a large batch needs more
    const size_t scratch = offsetof(F32Shared<D>, q) + (size_t)a.B * 12;
    static_assert(offsetof(F32Shared<D>, q) + (size_t)kAttnMaxB * 12 <= 227 * 1024 && sizeof(F32Shared<D>) <= 227 * 1024, "shared memory");
    const size_t smem = scratch > sizeof(F32Shared<D>) ? scratch : sizeof(F32Shared<D>);
    cudaError_t e = cudaSuccess;
    static std::atomic<uint64_t> prepared{0};
    int dev = 0;
    e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev > 63 || !(prepared.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(attention_f32_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
        if (e == cudaSuccess && dev <= 63) prepared.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (e == cudaSuccess) e = launch_behind(attention_f32_kernel<D>, dim3(kMaxBlocks), kF32Threads, smem, stream, a, ws);
    if (e == cudaSuccess)
        e = launch_behind(attention_combine_kernel<D, float>, dim3(kMaxBlocks, kCombineDims, kCombineRows), kCombineThreads, 0, stream, a, ws);
    return e;
}

}  // namespace

pcg_status attention_f32(const char *who, const AttnArgs &a, void *workspace, cudaStream_t stream) {
    const cudaError_t e = a.d == 128 ? launch<128>(a, workspace, stream) : launch<64>(a, workspace, stream);
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

}  // namespace pcg
