// What the kernels that write a key/value cache and read it back share (k_kv_cache.cu,
// k_kv4_cache.cu): rows of any type in vectors, which block a warp takes, the grid.
#pragma once
#include <algorithm>
#include <type_traits>

#include "skm_kv.cuh"

namespace skm {

namespace {

// Warps of a CTA: a block's keys and its values.  Warps end at different times, and their place is another's once their
// CTA has ended (with 8: 4-bit blocks read back 88 us for 82, written 71 for 68; 8-bit ones 101 for 96, 54 for 53)
constexpr int WARPS = 2;
template <typename T>
constexpr int WORDS8 = 8 * sizeof(T) / 4;  // words of 8 values

// 16 bytes without the alignment of a vector (not inlined: the loads would be
// predicated into the aligned path)
template <typename T>
__device__ __noinline__ uint4 load_slowly(const T *p) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
        for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
    } else {
        const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
        for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 8 consecutive values as they are
template <typename T>
__device__ __forceinline__ void load8(const T *p, int wide, uint32_t *w) {
#pragma unroll
    for (int i = 0; i < WORDS8<T>; i += 4) {
        const T *q = p + i * (4 / (int)sizeof(T));
        const uint4 a = wide ? *reinterpret_cast<const uint4 *>(q) : load_slowly(q);
        w[i] = a.x, w[i + 1] = a.y, w[i + 2] = a.z, w[i + 3] = a.w;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float *v) {
    if constexpr (std::is_same<T, float>::value) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Which block a warp takes: its sequence and how many blocks after the first.
// Up to 32 sequences, the blocks there are, in order; more, a row of
// most_blocks for each.
struct Place {
    int b, i;
};
__device__ __forceinline__ Place place_of(const KvCacheArgs &a, int u, int lane) {
    if (a.batch > 32) return Place{a.by_most.div(u), a.by_most.mod(u)};
    int n = 0;
    if (lane < a.batch) {
        const int2 rows = kv_rows_of(a.cu, lane, a.tokens, a.max_tokens);
        const int start = max(a.pos[lane], 0);
        if (rows.y > 0) n = (start % KV_B + rows.y + KV_B - 1) / KV_B;
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    const uint32_t after = __ballot_sync(0xffffffffu, x > u);  // the first whose blocks reach past u
    const int b = after ? __ffs(after) - 1 : a.batch;
    return Place{b, u - __shfl_sync(0xffffffffu, x - n, b & 31)};
}

// blocks that max_tokens rows reach at most, wherever the first one lies
int most_blocks_of(const KvCacheArgs &a) { return (int)(((int64_t)a.max_tokens + KV_B - 1 + KV_B - 1) / KV_B); }

// at most: the blocks of a row for each sequence, and those that the tokens fill and touch
int64_t grid_of(const KvCacheArgs &a) {
    int64_t blocks = (int64_t)a.batch * most_blocks_of(a);
    if (a.batch <= 32) blocks = std::min<int64_t>(blocks, a.tokens / KV_B + 2 * (int64_t)a.batch);
    return cdiv(blocks * a.heads * 2, WARPS);
}

KvCacheArgs with_divisions(KvCacheArgs a) {
    a.by_heads = FastDiv(a.heads);
    a.by_bpp = FastDiv(a.bpp);
    a.by_most = FastDiv(most_blocks_of(a));
    a.by_chunks = FastDiv(a.d / KV_B);
    a.by_eighths = FastDiv(a.d / 8);
    return a;
}

}  // namespace

#define KV_BY_TYPE(KERNEL, ...)                                                                             \
    do {                                                                                                    \
        if (dtype == SKM_DTYPE_F32) KERNEL<float __VA_OPT__(, ) __VA_ARGS__><<<grid, WARPS * 32, 0, st>>>(a); \
        else if (dtype == SKM_DTYPE_BF16)                                                                   \
            KERNEL<__nv_bfloat16 __VA_OPT__(, ) __VA_ARGS__><<<grid, WARPS * 32, 0, st>>>(a);               \
        else KERNEL<__half __VA_OPT__(, ) __VA_ARGS__><<<grid, WARPS * 32, 0, st>>>(a);                     \
    } while (0)

}  // namespace skm
