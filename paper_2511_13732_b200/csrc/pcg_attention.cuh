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
    float v_scale;       // (4 bits) what outputs are multiplied by
};

constexpr int kAttnMaxB = 16384, kAttnMaxGroup = 128;

// The kernels that share their work out among all SMs take head dimensions 64 and 128: the 16-bit types on the tensor
// cores, float32 on the FMA pipes.  Both need attention_work_bytes(d) of workspace.
inline bool attention_shares(int d) { return d == 64 || d == 128; }
size_t attention_work_bytes(int32_t d);
// What all attention calls refuse alike.
pcg_status check_attention(const char *who, const AttnArgs &a, pcg_dtype dtype, float scale);
pcg_status attention_tc(const char *who, const AttnArgs &a, pcg_dtype dtype, void *workspace, cudaStream_t stream);
pcg_status attention_f32(const char *who, const AttnArgs &a, void *workspace, cudaStream_t stream);

// Over the cache that holds 4.5 bits a value (k: its pages): 16-bit types, head dimensions 64 and 128, attention_work_bytes(d) of
// workspace.  Calls of few rows have a kernel of their own: `few_tile` says how many rows its row tiles are to have, for n tokens
// a sequence and G query heads a key head, 0 where the other kernel is the faster one.  (n = 4, 5 and 6, 7 and 8 of G = 4 over up
// to 8000, 64 sequences, 8 key heads x 128: 105, 165, 192 us, and 211 with the other; x 64: 73, 107, 132, and 168.
// Two tiles of 16 rows are faster than one of 32, whose sums no longer fit a lane's registers at head dimension 128, and three
// slower than the other kernel.)
inline int few_tile(int d, int64_t n, int G) {
    if (n * G <= (d == 64 ? 32 : 24)) return (int)n * G;
    return d == 128 && G <= 16 && n <= 2 * (16 / G) ? 16 : 0;
}
pcg_status attention_fourbit_few(const char *who, const AttnArgs &a, pcg_dtype dtype, int tile_rows, void *workspace, cudaStream_t stream);
pcg_status attention_fourbit_tc(const char *who, const AttnArgs &a, pcg_dtype dtype, int64_t rows, void *workspace, cudaStream_t stream);

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
