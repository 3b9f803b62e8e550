// Attention of packed rows over the cache that holds 4.5 bits a value (pcg_cache_attention_fourbit): the formulas are
// pcg_cache_attention's, over the values that codes and scales stand for.
#include <cuda_bf16.h>

#include <cmath>
#include <type_traits>

#include "pcg_attention.cuh"
#include "pcg_fourbit.cuh"

namespace pcg {

// ---------------------------------------------------------------------------------------------- float32, other head sizes
// One block per (row, query head): its eight warps take keys 32 at a time (two pages) in turn, a lane scores one key, and
// the warp sums the 32 weighted values with lane = head dimension, whose codes of a page are 8 bytes.  The warps'
// running sums meet in shared memory at the end.
// What bounds it: every key is read again for each row and each query head of its group, and products run on the FMA pipes.
// (64 single tokens of 32 query heads over up to 2000, 8 key heads, bfloat16: 139 us for 96 dimensions, 490 for 256.)
constexpr int kSimpleThreads = 256;

template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t narrow<uint16_t>(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
template <>
__device__ __forceinline__ f16_t narrow<f16_t>(float x) { return f16_t{__half_as_ushort(__float2half_rn(x))}; }

template <typename T, int DPL>  // DPL: values per lane, 32 * DPL = d
__global__ void __launch_bounds__(kSimpleThreads) attention_fourbit_simple_kernel(const __grid_constant__ AttnArgs a) {
    constexpr int NW = kSimpleThreads / 32, d = 32 * DPL;
    __shared__ float qs[d];
    __shared__ float part[NW][d + 2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = blockIdx.x, h = blockIdx.y, g = h / (a.q_heads / a.kv_heads);
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
    auto page_of = [&](int p) -> const uint8_t * {  // null: a block that stands for zeros
        const int32_t block = a.block_table[(int64_t)b * a.max_blocks + (p >> a.bs_shift)];
        if (block < 0 || block >= a.n_blocks) return nullptr;
        const int64_t in = (p & ((1 << a.bs_shift) - 1)) >> 4;
        return (const uint8_t *)a.k + ((((int64_t)block * a.kv_heads + g) << (a.bs_shift - 4)) + in) * page_bytes(d);
    };
    float m = kNegInf, l = 0.f, acc[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
    for (int p0 = warp * 32; p0 < lim; p0 += NW * 32) {
        const int p = p0 + lane;
        float s = kNegInf;
        if (p < lim) {
            s = 0.f;
            if (const uint8_t *page = page_of(p)) {
                const int tok = p & 15;
#pragma unroll 1
                for (int c = 0; c < d / 32; ++c) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(page + c * 256 + tok * 16);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float by = widen_scale(page[key_scales_at(d) + tok * (d / 16) + c * 2 + i / 2]);
                        uint32_t v[4];
                        widen_codes(w[i], v);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = both_halves(v[j]);
                            s = fmaf(f.x * by, qs[c * 32 + i * 8 + j * 2], s);
                            s = fmaf(f.y * by, qs[c * 32 + i * 8 + j * 2 + 1], s);
                        }
                    }
                }
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
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int k0 = p0 + half * 16, keys = min(16, lim - k0);
            if (keys <= 0) break;
            const uint8_t *page = page_of(k0);
            if (!page) continue;
#pragma unroll
            for (int i = 0; i < DPL; ++i) {
                const int dim = i * 32 + lane;
                const uint2 x = *reinterpret_cast<const uint2 *>(page + value_codes_at(d) + dim * 8);
                const uint4 sc = *reinterpret_cast<const uint4 *>(page + value_scales_at(d) + dim / 16 * 16);
                const uint32_t ws[4] = {sc.x, sc.y, sc.z, sc.w};
                uint32_t v[8], e[8];
                widen_codes(x.x, reinterpret_cast<uint32_t(&)[4]>(v[0]));
                widen_codes(x.y, reinterpret_cast<uint32_t(&)[4]>(v[4]));
#pragma unroll
                for (int j = 0; j < 4; ++j) widen_scales(ws[j], reinterpret_cast<uint32_t(&)[2]>(e[2 * j]));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 f = both_halves(v[j]), by = both_halves(e[j]);
                    const float w0 = __shfl_sync(0xffffffffu, w, half * 16 + 2 * j), w1 = __shfl_sync(0xffffffffu, w, half * 16 + 2 * j + 1);
                    if (2 * j < keys) acc[i] = fmaf(w0, f.x * by.x, acc[i]);  // what lies behind the last key may be anything
                    if (2 * j + 1 < keys) acc[i] = fmaf(w1, f.y * by.y, acc[i]);
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
    for (int i = 0; i < DPL; ++i) part[warp][i * 32 + lane] = acc[i];
    if (lane == 0) {
        part[warp][d] = m;
        part[warp][d + 1] = l;
    }
    __syncthreads();
    float top = kNegInf, total = 0.f;
    for (int w = 0; w < NW; ++w) top = fmaxf(top, part[w][d]);
    // a warp that has met no score above -inf has m = -inf and counts for nothing, unless one of its scores is NaN: its sum
    // of weights then is (0 otherwise), and so is the row
    for (int w = 0; w < NW; ++w) total += part[w][d + 1] * (part[w][d] != kNegInf ? exp2f(part[w][d] - top) : 0.f);
    T *out = (T *)a.out + ((int64_t)r * a.q_heads + h) * d;
    for (int i = tid; i < d; i += kSimpleThreads) {
        float o = 0.f;
        for (int w = 0; w < NW; ++w)
            if (part[w][d] != kNegInf) o += part[w][i] * exp2f(part[w][d] - top);
        out[i] = narrow<T>(lim > 0 ? o / total * a.v_scale : 0.f);
    }
}

template <typename T>
void launch_fourbit_simple(const AttnArgs &a, cudaStream_t s) {
    const dim3 grid(a.rows, a.q_heads);
    constexpr bool kAll = std::is_same<T, float>::value;  // 16-bit types have other kernels for 64 and 128 dimensions
    switch (a.d / 32) {
        case 1: attention_fourbit_simple_kernel<T, 1><<<grid, kSimpleThreads, 0, s>>>(a); break;
        case 2: if constexpr (kAll) attention_fourbit_simple_kernel<T, 2><<<grid, kSimpleThreads, 0, s>>>(a); break;
        case 3: attention_fourbit_simple_kernel<T, 3><<<grid, kSimpleThreads, 0, s>>>(a); break;
        case 4: if constexpr (kAll) attention_fourbit_simple_kernel<T, 4><<<grid, kSimpleThreads, 0, s>>>(a); break;
        case 5: attention_fourbit_simple_kernel<T, 5><<<grid, kSimpleThreads, 0, s>>>(a); break;
        case 6: attention_fourbit_simple_kernel<T, 6><<<grid, kSimpleThreads, 0, s>>>(a); break;
        case 7: attention_fourbit_simple_kernel<T, 7><<<grid, kSimpleThreads, 0, s>>>(a); break;
        default: attention_fourbit_simple_kernel<T, 8><<<grid, kSimpleThreads, 0, s>>>(a); break;
    }
}

}  // namespace pcg

using namespace pcg;

extern "C" pcg_status pcg_cache_attention_fourbit(const void *q, int64_t q_stride, pcg_dtype dtype, int32_t rows, int32_t q_heads,
                                                  const int32_t *row_start, const int32_t *kv_len, const int32_t *block_table,
                                                  int32_t B, int32_t max_blocks, const pcg_fourbit_cache *cache, float scale,
                                                  void *out, void *workspace, size_t workspace_bytes, pcg_stream stream) {
    const char *who = "pcg_cache_attention_fourbit";
    pcg_status st = check_fourbit(who, cache);
    if (st != PCG_OK) return st;
    if (!valid_dtype(dtype) || max_blocks < 1 || (int64_t)max_blocks * cache->block_size > 0x7fffff00) {
        set_error("%s: bad dtype %d, or max_blocks under 1, or max_blocks * block_size over 2^31 - 256 (got %d)", who, (int)dtype, max_blocks);
        return PCG_ERR_INVALID_ARG;
    }
    const AttnArgs a{q, cache->data, nullptr, out, row_start, kv_len, block_table, q_stride, 0, 0, rows, B, q_heads,
                     cache->kv_heads, cache->head_dim, max_blocks, cache->n_blocks, __builtin_ctz(cache->block_size),
                     scale * 1.4426950408889634f * cache->k_scale, 0, cache->v_scale};
    st = check_attention(who, a, dtype, scale);
    if (st == PCG_OK && !(a.scale_log2 > 0.f && std::isfinite(a.scale_log2))) {
        set_error("%s: the scale %g and the keys' %g have no product in float32", who, (double)scale, (double)cache->k_scale);
        st = PCG_ERR_INVALID_ARG;
    }
    if (st != PCG_OK || rows == 0 || B == 0) return st;
    if (!kv_len || !block_table) {
        set_error("%s: null pointer", who);
        return PCG_ERR_INVALID_ARG;
    }
    const size_t need = pcg_attention_workspace_bytes(B, q_heads, a.kv_heads, a.d, dtype);
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) {
        set_error("%s: the workspace must be 256-byte aligned and hold %zu bytes (got %zu)", who, need, workspace_bytes);
        return PCG_ERR_WORKSPACE;
    }
    st = check_here(who, out);
    if (st != PCG_OK) return st;
    if (dtype != PCG_F32 && (a.d == 64 || a.d == 128)) {
        // how many rows a sequence has is on the GPU: their average is known here
        const int64_t n = ((int64_t)rows + B - 1) / B;
        const int G = q_heads / a.kv_heads, few = few_tile(a.d, n, G);
        if (few) return attention_fourbit_few(who, a, dtype, few, workspace, (cudaStream_t)stream);
        return attention_fourbit_tc(who, a, dtype, n * G, workspace, (cudaStream_t)stream);
    }
    PCG_DISPATCH_DTYPE(dtype, launch_fourbit_simple<LogitT>(a, (cudaStream_t)stream));
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}
