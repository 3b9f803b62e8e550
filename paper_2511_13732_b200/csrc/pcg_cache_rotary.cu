// New keys and values into the cache with the rotation by position on the way, and into the cache that holds 4.5 bits a
// value; the queries of the same rows are turned by the same launch.
#include <cuda_bf16.h>

#include <cmath>

#include "pcg_fourbit.cuh"

namespace pcg {

// ---------------------------------------------------------------------------------------------- eight elements
template <typename T>
struct Eight {
    uint4 r[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);  // (read once)
    }
    __device__ __forceinline__ void store(T *p) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = r[i];
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {
        constexpr int N = Elem<T>::kPerVec;
#pragma unroll
        for (int i = 0; i < 8 / N; ++i) {
            float v[N];
            Elem<T>::unpack(r[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) x[i * N + j] = v[j];
        }
    }
    __device__ __forceinline__ void round(const float (&x)[8]);  // to nearest, ties to even
};
template <>
__device__ __forceinline__ void Eight<float>::round(const float (&x)[8]) {
    r[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    r[1] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
}
template <>
__device__ __forceinline__ void Eight<uint16_t>::round(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    r[0] = make_uint4(w[0], w[1], w[2], w[3]);
}
template <>
__device__ __forceinline__ void Eight<f16_t>::round(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    r[0] = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---------------------------------------------------------------------------------------------- rotation
struct Turn {
    const float *table;
    int32_t dim, interleaved, positions;
};

// Cosines and sines of pairs first .. first + N - 1 at a position; NaN where the table has no such position.
template <int N>
__device__ __forceinline__ void load_angles(const Turn &t, int pos, int first, float (&c)[N], float (&s)[N]) {
    if (pos < t.positions) {
        const float *row = t.table + (int64_t)pos * t.dim + first;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(row + i));
            const float4 b = __ldg(reinterpret_cast<const float4 *>(row + t.dim / 2 + i));
            c[i] = a.x, c[i + 1] = a.y, c[i + 2] = a.z, c[i + 3] = a.w;
            s[i] = b.x, s[i + 1] = b.y, s[i + 2] = b.z, s[i + 3] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = s[i] = __int_as_float(0x7fffffff);
    }
}
// One pair, each operation rounded by itself: the result does not depend on what the compiler would contract.
__device__ __forceinline__ void turn_pair(float &x1, float &x2, float c, float s) {
    const float y1 = __fsub_rn(__fmul_rn(x1, c), __fmul_rn(x2, s)), y2 = __fadd_rn(__fmul_rn(x2, c), __fmul_rn(x1, s));
    x1 = y1;
    x2 = y2;
}
// N elements each: pair i is (x1[i], x2[i]), or the pairs are adjacent, those of x1 first.
template <int N>
__device__ __forceinline__ void turn(float (&x1)[N], float (&x2)[N], const float (&c)[N], const float (&s)[N], bool adjacent) {
    if (adjacent) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            turn_pair(x1[2 * i], x1[2 * i + 1], c[i], s[i]);
            turn_pair(x2[2 * i], x2[2 * i + 1], c[N / 2 + i], s[N / 2 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) turn_pair(x1[i], x2[i], c[i], s[i]);
    }
}

struct RotaryArgs {
    const void *q, *k, *v;
    void *q_out, *k_out, *kc, *vc;
    const int32_t *slots, *positions;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride, n_slots;  // strides in elements
    int32_t rows, q_heads, kv_heads, d, bs_shift;
    Turn turn;
};

// A block is a row.  Its heads are cut into units of 8 pairs (16 elements); a thread keeps one unit's angles in registers and
// takes that unit of head after head, three heads at a time.  The first three and the first of its values are asked for
// before the row's position is known, which says whether they are needed and where the angles lie.  With `keys` also the
// keys, to the cache and k_out, and the values, which are copied.
// What bounds it: HBM -- 2 (q_heads + 2 kv_heads) head_dim elements a row.  (33,001 rows of 32 + 2 * 8 heads x 128 in bfloat16:
// 143 us, 89 % of the measured copy; heads asked for one at a time, behind the position, took 166.  4352 rows: 19 us.)
constexpr int kRotaryThreads = 128, kHeadsAtOnce = 3;

template <typename T>
__device__ __forceinline__ void rotary_row(const RotaryArgs &a, int64_t r, bool keys) {
    const int pos = a.positions[r];
    const int64_t slot = keys ? a.slots[r] : -1;
    const bool held = slot >= 0 && slot < a.n_slots;
    const int tid = threadIdx.x, d = a.d, dim = a.turn.dim, heads = a.q_heads + (keys ? a.kv_heads : 0);
    const T *q = (const T *)a.q + r * a.q_stride, *k = (const T *)a.k + r * a.k_stride, *v = (const T *)a.v + r * a.v_stride;
    auto get = [&](int h, int o, Eight<T> &x) { x.load(h < a.q_heads ? q + h * d + o : k + (h - a.q_heads) * d + o); };
    const int nu = dim / 16, step = kRotaryThreads / nu;  // units of a head; heads side by side
    const bool adjacent = a.turn.interleaved, turning = tid < step * nu;
    const int u = tid % nu, o1 = adjacent ? 16 * u : 8 * u, o2 = adjacent ? o1 + 8 : dim / 2 + o1;
    int h = turning ? tid / nu : heads;
    Eight<T> r1[kHeadsAtOnce], r2[kHeadsAtOnce], v0;
    auto ask = [&]() {
#pragma unroll
        for (int i = 0; i < kHeadsAtOnce; ++i)
            if (h + i * step < heads) {
                get(h + i * step, o1, r1[i]);
                get(h + i * step, o2, r2[i]);
            }
    };
    const int vecs = keys ? a.kv_heads * (d / 8) : 0;
    ask();
    if (tid < vecs) v0.load(v + tid * 8);
    if (pos < 0) return;
    const int64_t at = held ? (((slot >> a.bs_shift) * a.kv_heads) << a.bs_shift) + (slot & ((1 << a.bs_shift) - 1)) : 0;
    T *qo = (T *)a.q_out + r * a.q_out_stride, *ko = a.k_out ? (T *)a.k_out + r * a.k_out_stride : nullptr;
    // a head's rows in the cache are 1 << bs_shift apart
    auto cached = [&](void *cache, int h) { return (T *)cache + (at + ((int64_t)h << a.bs_shift)) * d; };
    auto put = [&](int h, int o, const Eight<T> &x) {
        if (h < a.q_heads) {
            x.store(qo + h * d + o);
        } else {
            if (held) x.store(cached(a.kc, h - a.q_heads) + o);
            if (ko) x.store(ko + (h - a.q_heads) * d + o);
        }
    };
    if (h < heads) {
        float c[8], s[8];
        load_angles<8>(a.turn, pos, 8 * u, c, s);
        while (true) {
#pragma unroll
            for (int i = 0; i < kHeadsAtOnce; ++i)
                if (h + i * step < heads) {
                    float x1[8], x2[8];
                    r1[i].widen(x1);
                    r2[i].widen(x2);
                    turn<8>(x1, x2, c, s, adjacent);
                    r1[i].round(x1);
                    r2[i].round(x2);
                    put(h + i * step, o1, r1[i]);
                    put(h + i * step, o2, r2[i]);
                }
            h += kHeadsAtOnce * step;
            if (h >= heads) break;
            ask();
        }
    }
    if (dim < d) {
        const int rest = (d - dim) / 8;
        for (int i = tid; i < heads * rest; i += kRotaryThreads) {
            const int h = i / rest, o = dim + (i - h * rest) * 8;
            Eight<T> x;
            get(h, o, x);
            put(h, o, x);
        }
    }
    if (held) {
        for (int i = tid; i < vecs; i += kRotaryThreads) {
            const int h = i / (d / 8), o = (i - h * (d / 8)) * 8;
            if (i != tid) v0.load(v + i * 8);
            v0.store(cached(a.vc, h) + o);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kRotaryThreads, sizeof(T) == 2 ? 8 : 4) cache_append_rotary_kernel(const __grid_constant__ RotaryArgs a) {
    rotary_row<T>(a, blockIdx.x, true);
}

// ---------------------------------------------------------------------------------------------- 4 bits
// 16 dimensions: their codes (dimension i in nibble i) and the scale.
__device__ __forceinline__ void quantise(float (&x)[16], float g, uint32_t (&code)[2], uint32_t &scale) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(x[i])), "f"(fabsf(x[i + 1])));
    uint16_t s8;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(s8) : "f"(0.f), "f"(__fdiv_rn(m, __fmul_rn(6.f, g))));
    scale = s8 & 0xffu;
    const float by = __fmul_rn(widen_scale(scale), g), inverse = __frcp_rn(by);
    if (m > 16.f * by) {  // a scale that ends at its largest value: beyond 16 codes do so too
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fminf(fmaxf(x[i], -16.f * by), 16.f * by);
    }
    const uint32_t some = scale == 0 ? 0u : 0xffffffffu;  // a scale of 0 holds zeros
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // x / by, as rounded as a division's: a product with the rounded reciprocal, and its remainder (exact in one fma) once
            // more (Markstein's correction; the signs so that -0 stays -0).  Remainders are far from float32's least values
            // wherever the quotient is near a border of two codes (a quarter at the least, by 2^-69 or more).
            const float z = x[8 * j + i], q = __fmul_rn(z, inverse);
            y[i] = __fmaf_rn(-__fmaf_rn(q, by, -z), inverse, q);
        }
        // (each byte widened to a register of its own: packed from four 8-bit registers and unpacked again by widen_codes, the
        // upper two came out 0 with the compiler of CUDA 12.9)
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm("{\n\t.reg .b8 a;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.u32.u8 %0, a;\n\t}" : "=r"(b[i]) : "f"(y[2 * i]), "f"(y[2 * i + 1]));
        code[j] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410) & some;
    }
}
// What is held of 8 of them: code * scale is exact, its product with the cache's scale rounded to float32, then to the type.
template <typename T>
__device__ __forceinline__ void store_held(T *p, uint32_t code, uint32_t scale, float g) {
    const float s = widen_scale(scale);
    uint32_t h[4];
    widen_codes(code, h);
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = both_halves(h[i]);
        x[2 * i] = __fmul_rn(__fmul_rn(f.x, s), g);
        x[2 * i + 1] = __fmul_rn(__fmul_rn(f.y, s), g);
    }
    Eight<T> r;
    r.round(x);
    r.store(p);
}

struct FourbitArgs {
    RotaryArgs r;  // kc: the cache's pages; without rotation turn.dim is 0
    void *v_out;
    float k_scale, v_scale;
};

// Blocks 0 .. windows * kv_heads - 1: the keys and values of one head of the rows that begin their page's part in one window
// of 16 rows.  A PART is a run of rows whose slots follow one another inside a page, as a sequence's do; a prompt's rows make
// whole pages of it, wherever they begin, and a round's make one part a sequence.  A thread quantises 32 dimensions of a
// token, keys by one half of the block and values by the other.  Key codes go straight to their place; value codes are turned
// through shared memory, a byte each, and written a dimension at a time: plainly where the part is the whole page, else
// the part's own nibbles by two atomics (and, or), since other rows of the call may write their neighbours.
// The other blocks turn the queries, a row each.
// What bounds it: 24,016 rows of 32 + 2 * 8 heads x 128 in bfloat16 take 134 us, 71 % of the measured copy: 68 of them the
// queries, near HBM's rate, and 66 the pages, where instructions (58 % of the issue slots) and the two barriers of a block
// alternate with its loads.  IEEE divisions instead of the product with the reciprocal took 191 in all; blocks that take several
// heads of a window with the next one's loads under way 137, the two kinds of blocks mixed evenly 139 (their code then shares
// the instruction caches), rotation and quotients on pairs of float32 at once 131 to 134 but 1 us more for the append above.
constexpr int kFourbitThreads = kRotaryThreads;

template <typename T>
__global__ void __launch_bounds__(kFourbitThreads, sizeof(T) == 2 ? 8 : 4) cache_append_fourbit_kernel(const __grid_constant__ FourbitArgs f, int windows) {
    extern __shared__ __align__(16) uint8_t codes[];  // [32][d + 16]: value codes of the rows, a byte each
    __shared__ int32_t slot_of[32];
    __shared__ uint32_t begins;
    const RotaryArgs &a = f.r;
    const int64_t page_blocks = (int64_t)windows * a.kv_heads;
    if (blockIdx.x >= page_blocks) {
        rotary_row<T>(a, blockIdx.x - page_blocks, false);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = a.d, pitch = d + 16;
    const int h = blockIdx.x % a.kv_heads;
    const int64_t r0 = (int64_t)(blockIdx.x / a.kv_heads) * 16;
    // the slots of the window's rows and of the next one's: -1 outside the cache, -2 a row that has no part in the call
    auto slot_at = [&](int64_t r) -> int32_t {
        if (r < 0 || r >= a.rows || (a.positions && a.positions[r] < 0)) return -2;
        const int32_t s = a.slots[r];
        return s < 0 || s >= a.n_slots ? -1 : s;
    };
    if (warp == 0) {
        const int32_t s = slot_at(r0 + lane), before = lane == 0 ? slot_at(r0 - 1) : 0;
        int32_t prev = __shfl_up_sync(0xffffffffu, s, 1);
        if (lane == 0) prev = before;
        slot_of[lane] = s;
        const uint32_t mask = __ballot_sync(0xffffffffu, s < 0 || prev < 0 || s != prev + 1 || (s & 15) == 0);
        if (lane == 0) begins = mask;
    }
    __syncthreads();
    if ((begins & 0xffffu) == 0) return;
    // a part has at most 16 rows, so the next window's first part begins among the 32
    const int lo = __ffs(begins) - 1, hi = (begins >> 16) ? __ffs(begins >> 16) + 15 : 32;
    const int nu = d / 32, half = kFourbitThreads / 2, t = tid & (half - 1), tokens = half / nu;
    const bool keys = tid < half;
    if (t < tokens * nu) {
        const int u = t % nu;
        const bool turned = keys && u < a.turn.dim / 32, adjacent = a.turn.interleaved;
        const int o1 = turned && !adjacent ? 16 * u : 32 * u, o2 = turned && !adjacent ? a.turn.dim / 2 + o1 : o1 + 16;
        const float g = keys ? f.k_scale : f.v_scale;
        for (int i = lo + t / nu; i < hi; i += tokens) {
            const int32_t slot = slot_of[i];
            const int64_t r = r0 + i;
            if (slot == -2) continue;
            const T *src = keys ? (const T *)a.k + r * a.k_stride + h * d : (const T *)a.v + r * a.v_stride + h * d;
            Eight<T> raw[4];
            raw[0].load(src + o1);
            raw[1].load(src + o1 + 8);
            raw[2].load(src + o2);
            raw[3].load(src + o2 + 8);
            float x[2][16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float y[8];
                raw[j].widen(y);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j >> 1][(j & 1) * 8 + e] = y[e];
            }
            if (turned) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {  // (registers)
                    float c[8], s[8], x1[8], x2[8];
                    load_angles<8>(a.turn, a.positions[r], 16 * u + 8 * half, c, s);
                    // adjacent: pairs 8 half .. of the 16 lie in one group; else across the two
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x1[e] = adjacent ? x[half][e] : x[0][8 * half + e];
                        x2[e] = adjacent ? x[half][8 + e] : x[1][8 * half + e];
                    }
                    turn<8>(x1, x2, c, s, adjacent);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (adjacent) {
                            x[half][e] = x1[e];
                            x[half][8 + e] = x2[e];
                        } else {
                            x[0][8 * half + e] = x1[e];
                            x[1][8 * half + e] = x2[e];
                        }
                    }
                }
            }
            T *out = (T *)(keys ? a.k_out : f.v_out);
            uint8_t *page = (uint8_t *)a.kc;
            int tok = 0;
            if (slot >= 0) {
                tok = slot & 15;
                const int64_t block = slot >> a.bs_shift, in = (slot & ((1 << a.bs_shift) - 1)) >> 4;
                page += (((block * a.kv_heads + h) << (a.bs_shift - 4)) + in) * page_bytes(d);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int o = j ? o2 : o1;
                uint32_t code[2], scale;
                quantise(x[j], g, code, scale);
                if (out) {
                    T *to = out + (r * a.kv_heads + h) * d + o;
                    store_held<T>(to, code[0], scale, g);
                    store_held<T>(to + 8, code[1], scale, g);
                }
                if (slot < 0) continue;
                if (keys) {
                    *reinterpret_cast<uint2 *>(page + o / 32 * 256 + tok * 16 + (o & 16) / 2) = make_uint2(code[0], code[1]);
                    page[key_scales_at(d) + tok * (d / 16) + o / 16] = (uint8_t)scale;
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t low = code[e] & 0x0f0f0f0fu, high = (code[e] >> 4) & 0x0f0f0f0fu;
                        w[2 * e] = __byte_perm(low, high, 0x5140);
                        w[2 * e + 1] = __byte_perm(low, high, 0x7362);
                    }
                    *reinterpret_cast<uint4 *>(codes + i * pitch + o) = make_uint4(w[0], w[1], w[2], w[3]);
                    page[value_scales_at(d) + o + tok] = (uint8_t)scale;
                }
            }
        }
    }
    __syncthreads();
    // parts, a warp each in turn; a lane has four dimensions
    uint32_t mask = begins;
    for (int n = 0; mask; ++n) {
        const int i = __ffs(mask) - 1;
        mask &= mask - 1;
        if (i >= hi) break;
        const int end = mask ? __ffs(mask) - 1 : 32, slot = slot_of[i];
        if (slot < 0 || (n & 3) != warp) continue;
        const int t0 = slot & 15, len = end - i;
        const int64_t block = slot >> a.bs_shift, in = (slot & ((1 << a.bs_shift) - 1)) >> 4;
        uint8_t *page = (uint8_t *)a.kc + (((block * a.kv_heads + h) << (a.bs_shift - 4)) + in) * page_bytes(d) + value_codes_at(d);
        for (int o = lane * 4; o < d; o += 128) {
            uint32_t x[8];  // byte j of x[p]: tokens 2 p and 2 p + 1 of dimension o + j
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                x[p] = 0;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = 2 * p + e - t0;
                    if (at >= 0 && at < len) x[p] |= *reinterpret_cast<const uint32_t *>(codes + (i + at) * pitch + o) << (4 * e);
                }
            }
            uint32_t w[4][2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {  // 4 x 4 bytes turned
                const uint32_t ab = __byte_perm(x[4 * e], x[4 * e + 1], 0x5140), cd = __byte_perm(x[4 * e + 2], x[4 * e + 3], 0x5140);
                const uint32_t ef = __byte_perm(x[4 * e], x[4 * e + 1], 0x7362), gh = __byte_perm(x[4 * e + 2], x[4 * e + 3], 0x7362);
                w[0][e] = __byte_perm(ab, cd, 0x5410);
                w[1][e] = __byte_perm(ab, cd, 0x7632);
                w[2][e] = __byte_perm(ef, gh, 0x5410);
                w[3][e] = __byte_perm(ef, gh, 0x7632);
            }
            if (len == 16) {
                reinterpret_cast<uint4 *>(page + o * 8)[0] = make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
                reinterpret_cast<uint4 *>(page + o * 8)[1] = make_uint4(w[2][0], w[2][1], w[3][0], w[3][1]);
            } else {
                const unsigned long long own = ((1ull << (4 * len)) - 1) << (4 * t0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    unsigned long long *to = reinterpret_cast<unsigned long long *>(page + (o + j) * 8);
                    atomicAnd(to, ~own);
                    atomicOr(to, (unsigned long long)w[j][1] << 32 | w[j][0]);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- host
pcg_status check_fourbit(const char *who, const pcg_fourbit_cache *c) {
    if (!c || !c->data || ((uintptr_t)c->data & 15u)) {
        set_error("%s: the cache is null, or its data null or not 16-byte aligned", who);
        return PCG_ERR_INVALID_ARG;
    }
    constexpr float kLeast = 0x1p-60f, kMost = 0x1p60f;
    if (!valid_block_size(c->block_size) || c->n_blocks < 1 || c->kv_heads < 1 || c->kv_heads > 1024 || c->head_dim < 32 ||
        c->head_dim > 256 || c->head_dim % 32 || (int64_t)c->n_blocks * c->block_size > 0x7fffffff ||
        !(c->k_scale >= kLeast && c->k_scale <= kMost && c->v_scale >= kLeast && c->v_scale <= kMost)) {
        set_error("%s: bad cache (%d blocks of %d tokens, %d heads of %d, scales %g and %g): block_size is 16, 32, 64, 128 or 256, "
                  "head_dim a multiple of 32 up to 256, kv_heads 1 to 1024, scales 2^-60 to 2^60, and the slots fit 31 bits",
                  who, c->n_blocks, c->block_size, c->kv_heads, c->head_dim, (double)c->k_scale, (double)c->v_scale);
        return PCG_ERR_INVALID_ARG;
    }
    return PCG_OK;
}

namespace {

pcg_status check_rotary(const char *who, const pcg_rotary *t, int32_t d, int32_t multiple) {
    if (!t || !t->table || ((uintptr_t)t->table & 15u) || t->positions < 1 || t->dim < multiple || t->dim > d || t->dim % multiple ||
        (t->interleaved != 0 && t->interleaved != 1)) {
        set_error("%s: the rotation is null, its table null, empty or not 16-byte aligned, or its dim not a multiple of %d up to "
                  "head_dim", who, multiple);
        return PCG_ERR_INVALID_ARG;
    }
    return PCG_OK;
}

// q and q_out: both there or both not.
pcg_status check_queries(const char *who, const RotaryArgs &a, pcg_dtype dtype) {
    if (a.q_heads < 0 || a.q_heads > 65535 || (a.q_heads > 0) != (a.q != nullptr) || (a.q != nullptr) != (a.q_out != nullptr)) {
        set_error("%s: q, q_out and q_heads go together (q_heads=%d)", who, a.q_heads);
        return PCG_ERR_INVALID_ARG;
    }
    if (!a.q) return PCG_OK;
    if (a.q == a.q_out && a.q_stride != a.q_out_stride) {
        set_error("%s: queries that are turned in place keep their stride", who);
        return PCG_ERR_INVALID_ARG;
    }
    pcg_status st = check_rows(who, "q", a.q, a.q_stride, a.q_heads, a.d, dtype);
    return st != PCG_OK ? st : check_rows(who, "q_out", a.q_out, a.q_out_stride, a.q_heads, a.d, dtype);
}

}  // namespace
}  // namespace pcg

using namespace pcg;

extern "C" pcg_status pcg_cache_append_rotary(const void *q, int64_t q_stride, int32_t q_heads, const void *k, int64_t k_stride,
                                              const void *v, int64_t v_stride, int32_t rows, const int32_t *slots,
                                              const int32_t *positions, const pcg_rotary *rotary, const pcg_cache *cache,
                                              void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride,
                                              pcg_stream stream) {
    const char *who = "pcg_cache_append_rotary";
    pcg_status st = check_cache(who, cache);
    if (st == PCG_OK) st = check_rotary(who, rotary, cache->head_dim, 16);
    if (st != PCG_OK) return st;
    if (rows < 0 || (rows > 0 && (!slots || !positions))) {
        set_error("%s: rows < 0, or null slots or positions", who);
        return PCG_ERR_INVALID_ARG;
    }
    if (rows == 0) return PCG_OK;
    const RotaryArgs a{q, k, v, q_out, k_out, cache->k, cache->v, slots, positions, q_stride, k_stride, v_stride, q_out_stride,
                       k_out_stride, (int64_t)cache->n_blocks * cache->block_size, rows, q_heads, cache->kv_heads, cache->head_dim,
                       __builtin_ctz(cache->block_size), {rotary->table, rotary->dim, rotary->interleaved, rotary->positions}};
    st = check_queries(who, a, cache->dtype);
    if (st == PCG_OK) st = check_rows(who, "k", k, k_stride, a.kv_heads, a.d, cache->dtype);
    if (st == PCG_OK) st = check_rows(who, "v", v, v_stride, a.kv_heads, a.d, cache->dtype);
    if (st == PCG_OK && k_out) st = check_rows(who, "k_out", k_out, k_out_stride, a.kv_heads, a.d, cache->dtype);
    if (st == PCG_OK && k_out == k && k_out_stride != k_stride) {
        set_error("%s: keys that are turned in place keep their stride", who);
        st = PCG_ERR_INVALID_ARG;
    }
    if (st == PCG_OK) st = check_here(who, cache->k);
    if (st != PCG_OK) return st;
    PCG_DISPATCH_DTYPE(cache->dtype, cache_append_rotary_kernel<LogitT><<<rows, kRotaryThreads, 0, (cudaStream_t)stream>>>(a));
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}

extern "C" pcg_status pcg_cache_append_fourbit(const void *q, int64_t q_stride, int32_t q_heads, const void *k, int64_t k_stride,
                                               const void *v, int64_t v_stride, pcg_dtype dtype, int32_t rows,
                                               const int32_t *slots, const int32_t *positions, const pcg_rotary *rotary,
                                               const pcg_fourbit_cache *cache, void *q_out, int64_t q_out_stride, void *k_out,
                                               void *v_out, pcg_stream stream) {
    const char *who = "pcg_cache_append_fourbit";
    pcg_status st = check_fourbit(who, cache);
    if (st == PCG_OK && rotary) st = check_rotary(who, rotary, cache->head_dim, 32);
    if (st != PCG_OK) return st;
    if (!valid_dtype(dtype) || rows < 0 || (rows > 0 && (!slots || (rotary && !positions)))) {
        set_error("%s: bad dtype %d, rows < 0, or null slots or positions", who, (int)dtype);
        return PCG_ERR_INVALID_ARG;
    }
    if (!rotary && (q || q_out || q_heads)) {
        set_error("%s: queries without a rotation", who);
        return PCG_ERR_INVALID_ARG;
    }
    if (rows == 0) return PCG_OK;
    FourbitArgs f{{q, k, v, q_out, k_out, cache->data, nullptr, slots, rotary ? positions : nullptr, q_stride, k_stride, v_stride,
                   q_out_stride, 0, (int64_t)cache->n_blocks * cache->block_size, rows, q_heads, cache->kv_heads, cache->head_dim,
                   __builtin_ctz(cache->block_size), {nullptr, 0, 0, 0}}, v_out, cache->k_scale, cache->v_scale};
    if (rotary) f.r.turn = Turn{rotary->table, rotary->dim, rotary->interleaved, rotary->positions};
    const RotaryArgs &a = f.r;
    st = check_queries(who, a, dtype);
    if (st == PCG_OK) st = check_rows(who, "k", k, k_stride, a.kv_heads, a.d, dtype);
    if (st == PCG_OK) st = check_rows(who, "v", v, v_stride, a.kv_heads, a.d, dtype);
    if (st == PCG_OK && (((uintptr_t)k_out | (uintptr_t)v_out) & 15u)) {
        set_error("%s: k_out or v_out is not 16-byte aligned", who);
        st = PCG_ERR_INVALID_ARG;
    }
    const int64_t windows = ((int64_t)rows + 15) / 16, grid = windows * a.kv_heads + (q ? rows : 0);
    if (st == PCG_OK && grid > 0x7fffffff) {
        set_error("%s: %d rows of %d heads are more than a launch holds", who, rows, a.kv_heads);
        st = PCG_ERR_UNSUPPORTED;
    }
    if (st == PCG_OK) st = check_here(who, cache->data);
    if (st != PCG_OK) return st;
    const size_t smem = (size_t)32 * (a.d + 16);
    PCG_DISPATCH_DTYPE(dtype, cache_append_fourbit_kernel<LogitT><<<(unsigned)grid, kFourbitThreads, smem, (cudaStream_t)stream>>>(f, (int)windows));
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PCG_OK : cuda_fail(e, who);
}
