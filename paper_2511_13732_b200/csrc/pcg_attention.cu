// Attention of packed rows, causal inside each sequence's new rows: over a paged key/value cache (pcg_cache_attention)
// and over the rows' own keys and values (pcg_prompt_attention).
//     o_i = sum_{p < lim_i} w_p v_p / sum_{p < lim_i} w_p,   w_p = 2^(c (q_i . k_p) - m),   c = scale * log2 e,
// with one pass over the keys: m is a running reference, and what has been summed is scaled when it moves.
#include <cuda_bf16.h>

#include <cmath>

#include "pcg_attention.cuh"

namespace pcg {

// Rounding a float to the element type (nearest even), once.
template <typename T>
struct Narrow;
template <>
struct Narrow<float> {
    static __device__ __forceinline__ void store(float *p, float x) { *p = x; }
};
template <>
struct Narrow<uint16_t> {
    static __device__ __forceinline__ void store(uint16_t *p, float x) { *p = __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
};
template <>
struct Narrow<f16_t> {
    static __device__ __forceinline__ void store(f16_t *p, float x) { p->bits = __half_as_ushort(__float2half_rn(x)); }
};

// ---------------------------------------------------------------------------------------------- any type and head size
// One block per (row, query head): its eight warps take keys 32 at a time in turn, a lane scores one key (16-byte loads,
// the query in shared memory), and the warp sums the 32 weighted values with lane = head dimension.  The warps'
// running sums meet in shared memory at the end.  Serves the head dimensions that the other kernels are not built for.
// What bounds it: every key is read again, out of L2, for each row and each query head of its group, and products run on the
// FMA pipes: 2.3 to 4.9 TFLOP/s.  64 tokens over 2000 cached, 32 / 8 heads, bf16: 560 us at 80 dimensions, 1072 at 256 (118 at
// 128, on the tensor cores); a prompt of 2048: 6.4 ms, 15.0 ms (0.083 ms).  float16 above 64 dimensions spills 12 to 24 bytes
// a thread.
constexpr int kSimpleThreads = 256;

template <typename T, int DPL>  // DPL: values per lane, 32 * DPL >= d
__global__ void __launch_bounds__(kSimpleThreads) attention_simple_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int NW = kSimpleThreads / 32, PV = Elem<T>::kPerVec;
    __shared__ float qs[256];
    __shared__ float part[NW][32 * DPL + 2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = blockIdx.x, h = blockIdx.y, g = h / (a.q_heads / a.kv_heads), d = a.d;
    int lo = 0, hi = a.B - 1;  // the last sequence that starts at or before row r
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.row_start[mid] <= r)
            lo = mid;
        else
            hi = mid - 1;
    }
    const int b = lo;
    int begin, n, len;
    attn_sequence(a, b, begin, n, len);
    if (r < begin || r >= begin + n) return;  // belongs to no sequence: left as it is
    const int lim = len - n + (r - begin) + 1;
    const T *q = (const T *)a.q + (int64_t)r * a.q_stride + (int64_t)h * d;
    for (int i = tid; i < d; i += kSimpleThreads) qs[i] = Elem<T>::widen(q[i]) * a.scale_log2;
    __syncthreads();
    // element offsets of token p's row in the key and value arrays; false: a block that stands for zeros
    auto token = [&](int p, int64_t &ko, int64_t &vo) -> bool {
        if (!a.kv_len) {
            const int64_t t = (int64_t)begin + p;
            ko = t * a.k_stride + (int64_t)g * d;
            vo = t * a.v_stride + (int64_t)g * d;
            return true;
        }
        const int32_t block = a.block_table[(int64_t)b * a.max_blocks + (p >> a.bs_shift)];
        if (block < 0 || block >= a.n_blocks) return false;
        ko = vo = ((((int64_t)block * a.kv_heads + g) << a.bs_shift) + (p & ((1 << a.bs_shift) - 1))) * d;
        return true;
    };
    float m = kNegInf, l = 0.f, acc[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
    for (int p0 = warp * 32; p0 < lim; p0 += NW * 32) {
        const int p = p0 + lane;
        float s = kNegInf;
        int64_t ko = 0, vo = -1;
        if (p < lim) {
            s = 0.f;
            if (token(p, ko, vo)) {
                const uint4 *k = reinterpret_cast<const uint4 *>((const T *)a.k + ko);
                float s1 = 0.f;
                for (int c = 0; c < d / PV; ++c) {
                    float kv[PV];
                    Elem<T>::unpack(k[c], kv);
#pragma unroll
                    for (int i = 0; i < PV; i += 2) {
                        s = fmaf(kv[i], qs[c * PV + i], s);
                        s1 = fmaf(kv[i + 1], qs[c * PV + i + 1], s1);
                    }
                }
                s += s1;
            }
        }
        float top = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (top > m) {  // warp-uniform
            const float f = exp2f(m - top);  // 0 the first time
            l *= f;
#pragma unroll
            for (int i = 0; i < DPL; ++i) acc[i] *= f;
            m = top;
        }
        // a key behind the row's limit has s = -inf and weighs 0, as does a score of -inf in its place, whatever m is;
        // a row of such scores alone ends with 0 / 0 = NaN, as its softmax does
        const float w = s == kNegInf ? 0.f : exp2f(s - m);
        l += w;
        const int keys = min(32, lim - p0);
        for (int j = 0; j < keys; ++j) {
            const float wj = __shfl_sync(0xffffffffu, w, j);
            const int64_t o = __shfl_sync(0xffffffffu, vo, j);
            if (o < 0) continue;
            const T *v = (const T *)a.v + o;
#pragma unroll
            for (int i = 0; i < DPL; ++i)
                if (i * 32 + lane < d) acc[i] = fmaf(wj, Elem<T>::widen(v[i * 32 + lane]), acc[i]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
    for (int i = 0; i < DPL; ++i) part[warp][i * 32 + lane] = acc[i];
    if (lane == 0) {
        part[warp][32 * DPL] = m;
        part[warp][32 * DPL + 1] = l;
    }
    __syncthreads();
    float top = kNegInf, total = 0.f;
    for (int w = 0; w < NW; ++w) top = fmaxf(top, part[w][32 * DPL]);
    // a warp that has met no score above -inf has m = -inf and counts for nothing, unless one of its scores is NaN: its sum
    // of weights then is (0 otherwise), and so is the row
    for (int w = 0; w < NW; ++w) total += part[w][32 * DPL + 1] * (part[w][32 * DPL] != kNegInf ? exp2f(part[w][32 * DPL] - top) : 0.f);
    T *out = (T *)a.out + ((int64_t)r * a.q_heads + h) * d;
    for (int i = tid; i < d; i += kSimpleThreads) {
        float o = 0.f;
        for (int w = 0; w < NW; ++w)
            if (part[w][32 * DPL] != kNegInf) o += part[w][i] * exp2f(part[w][32 * DPL] - top);
        Narrow<T>::store(out + i, lim > 0 ? o / total : 0.f);
    }
}

template <typename T>
void launch_simple(const AttnArgs &a, cudaStream_t s) {
    const dim3 grid(a.rows, a.q_heads);
    if (a.d <= 64)
        attention_simple_kernel<T, 2><<<grid, kSimpleThreads, 0, s>>>(a);
    else if (a.d <= 128)
        attention_simple_kernel<T, 4><<<grid, kSimpleThreads, 0, s>>>(a);
    else
        attention_simple_kernel<T, 8><<<grid, kSimpleThreads, 0, s>>>(a);
}

pcg_status run_attention(const char *who, const AttnArgs &a, pcg_dtype dtype, void *workspace, size_t workspace_bytes,
                         cudaStream_t stream) {
    const size_t need = pcg_attention_workspace_bytes(a.B, a.q_heads, a.kv_heads, a.d, dtype);
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes (got %zu)", who, need, workspace_bytes);
        return PCG_ERR_WORKSPACE;
    }
    pcg_status st = check_here(who, a.out);
    if (st != PCG_OK) return st;
    if (attention_shares(a.d))
        return dtype == PCG_F32 ? attention_f32(who, a, workspace, stream) : attention_tc(who, a, dtype, workspace, stream);
    PCG_DISPATCH_DTYPE(dtype, launch_simple<LogitT>(a, stream));
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

// What both calls refuse alike.
pcg_status check_attention(const char *who, const AttnArgs &a, pcg_dtype dtype, float scale) {
    if (a.rows < 0 || a.B < 0 || a.q_heads < 1 || a.kv_heads < 1 || a.q_heads % a.kv_heads || a.q_heads > 65535 ||
        !(scale > 0.f) || !std::isfinite(scale)) {
        set_error("%s: need rows, B >= 0, q_heads a multiple of kv_heads, and a finite scale > 0 (rows=%d B=%d q_heads=%d "
                  "kv_heads=%d scale=%g)", who, a.rows, a.B, a.q_heads, a.kv_heads, (double)scale);
        return PCG_ERR_INVALID_ARG;
    }
    if (a.B > kAttnMaxB || a.q_heads / a.kv_heads > kAttnMaxGroup) {
        set_error("%s: B=%d and %d query heads a key head: at most %d and %d are supported", who, a.B,
                  a.q_heads / a.kv_heads, kAttnMaxB, kAttnMaxGroup);
        return PCG_ERR_UNSUPPORTED;
    }
    if (a.rows == 0 || a.B == 0) return PCG_OK;
    if (!a.row_start || !a.out || ((uintptr_t)a.out & 15u)) {
        set_error("%s: null pointer, or out is not 16-byte aligned", who);
        return PCG_ERR_INVALID_ARG;
    }
    return check_rows(who, "q", a.q, a.q_stride, a.q_heads, a.d, dtype);
}

}  // namespace pcg

using namespace pcg;

extern "C" size_t pcg_attention_workspace_bytes(int32_t B, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                                pcg_dtype dtype) {
    return attention_shares(head_dim) ? attention_work_bytes(head_dim) : 256;
}

extern "C" pcg_status pcg_cache_attention(const void *q, int64_t q_stride, int32_t rows, int32_t q_heads,
                                          const int32_t *row_start, const int32_t *kv_len, const int32_t *block_table,
                                          int32_t B, int32_t max_blocks, const pcg_cache *cache, float scale, void *out,
                                          void *workspace, size_t workspace_bytes, pcg_stream stream) {
    const char *who = "pcg_cache_attention";
    pcg_status st = check_cache(who, cache);
    if (st != PCG_OK) return st;
    if (max_blocks < 1 || (int64_t)max_blocks * cache->block_size > 0x7fffff00) {  // a key tile's end fits 31 bits
        set_error("%s: max_blocks must be at least 1, and max_blocks * block_size at most 2^31 - 256 (got %d)", who, max_blocks);
        return PCG_ERR_INVALID_ARG;
    }
    const AttnArgs a{q, cache->k, cache->v, out, row_start, kv_len, block_table, q_stride, 0, 0, rows, B, q_heads,
                     cache->kv_heads, cache->head_dim, max_blocks, cache->n_blocks, __builtin_ctz(cache->block_size),
                     scale * 1.4426950408889634f, 0};
    st = check_attention(who, a, cache->dtype, scale);
    if (st != PCG_OK || rows == 0 || B == 0) return st;
    if (!kv_len || !block_table) {
        set_error("%s: null pointer", who);
        return PCG_ERR_INVALID_ARG;
    }
    return run_attention(who, a, cache->dtype, workspace, workspace_bytes, (cudaStream_t)stream);
}

extern "C" pcg_status pcg_prompt_attention(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                                           int64_t v_stride, pcg_dtype dtype, int32_t rows, int32_t q_heads,
                                           int32_t kv_heads, int32_t head_dim, const int32_t *row_start, int32_t B,
                                           float scale, void *out, void *workspace, size_t workspace_bytes,
                                           pcg_stream stream) {
    const char *who = "pcg_prompt_attention";
    if (!valid_dtype(dtype) || head_dim < 8 || head_dim > 256 || head_dim % 8 || kv_heads > 1024) {
        set_error("%s: bad dtype %d, head_dim %d (a multiple of 8 up to 256) or kv_heads %d (up to 1024)", who, (int)dtype,
                  head_dim, kv_heads);
        return PCG_ERR_INVALID_ARG;
    }
    const AttnArgs a{q, k, v, out, row_start, nullptr, nullptr, q_stride, k_stride, v_stride, rows, B, q_heads, kv_heads,
                     head_dim, 0, 0, 0, scale * 1.4426950408889634f, 0};
    pcg_status st = check_attention(who, a, dtype, scale);
    if (st != PCG_OK || rows == 0 || B == 0) return st;
    st = check_rows(who, "k", k, k_stride, kv_heads, head_dim, dtype);
    if (st == PCG_OK) st = check_rows(who, "v", v, v_stride, kv_heads, head_dim, dtype);
    if (st != PCG_OK) return st;
    return run_attention(who, a, dtype, workspace, workspace_bytes, (cudaStream_t)stream);
}
