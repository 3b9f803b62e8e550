// What the attention kernels share: their arguments, the split of the work, the tensor-core path's entry.
#pragma once

#include "pcg_cache.cuh"

namespace pcg {

struct AttnArgs {
    const void *q, *k, *v;  // k, v: the cache's arrays, or the packed rows
    void *out;
    const int32_t *row_start, *kv_len, *block_table;  // kv_len null: the packed rows are the keys
    int64_t q_stride, k_stride, v_stride;  // elements between tokens (k, v: packed rows only)
    int32_t rows, B, q_heads, kv_heads, d;
    int32_t max_blocks, n_blocks, bs_shift;
    float scale_log2;
    int32_t few_tokens;  // (tensor cores) tokens of one copy of an item with one row tile
};

constexpr int kAttnMaxB = 16384, kAttnMaxGroup = 128;

// The kernels that share their work out among all SMs take head dimensions 64 and 128: the 16-bit types on the tensor
// cores, float32 on the FMA pipes.  Both need attention_work_bytes(d) of workspace.
inline bool attention_shares(int d) { return d == 64 || d == 128; }
size_t attention_work_bytes(int32_t d);
pcg_status attention_tc(const char *who, const AttnArgs &a, pcg_dtype dtype, void *workspace, cudaStream_t stream);
pcg_status attention_f32(const char *who, const AttnArgs &a, void *workspace, cudaStream_t stream);

#ifdef __CUDACC__

// Rows of sequence b, cut to the packed rows whatever row_start holds, and the keys that its last row may see.
__device__ __forceinline__ void attn_sequence(const AttnArgs &a, int b, int &begin, int &n, int &len) {
    begin = min(max(a.row_start[b], 0), a.rows);
    n = max(min(a.row_start[b + 1], a.rows) - begin, 0);
    len = n;
    if (a.kv_len) {
        const int64_t room = (int64_t)a.max_blocks << a.bs_shift;
        len = (int)min((int64_t)max(a.kv_len[b], 0), room);
    }
}

#endif  // __CUDACC__

}  // namespace pcg
