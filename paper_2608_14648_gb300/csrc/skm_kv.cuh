// Key/value caches and rotary positions: shared by the kernels (k_kv_*.cu) and their entry
// points (skm_kv.cu).
#pragma once
#include <atomic>

#include <cuda_fp16.h>

#include "skm_internal.cuh"

namespace skm {

constexpr int KV_B = SKM_KV_BLOCK;
constexpr int KV_SMS = 152;
// bytes of a 4-bit block: the codes of 16 keys and values, 16 x (scale, bias) of both in f16
__host__ __device__ __forceinline__ constexpr int kv4_bytes(int d) { return KV_B * d + 8 * KV_B; }
// sequences whose prefix sums one launch keeps in shared memory at most; larger
// batches take several launches
constexpr int KV_MAX_SEQS = 1024;

// n / d for 0 <= n < 2^31 without a division (the divisors of a launch: a
// division is a chain of some 40 dependent instructions): Granlund and Montgomery, Division by
// invariant integers using multiplication, PLDI 1994
struct FastDiv {
    uint32_t d, mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t n) : d(n), shift(0) {
        while ((uint64_t(1) << shift) < n) ++shift;
        mul = (uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << shift) - n)) / n + 1);
    }
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift); }
    __device__ __forceinline__ int mod(int n) const { return n - div(n) * (int)d; }
};

struct KvTokens {
    const void *x;
    int64_t token, head;  // strides, elements
    int wide;             // 16-byte vectors of it are aligned
};

struct KvCacheArgs {
    uint8_t *k, *v;
    float2 *scales;
    const int32_t *table, *pos, *cu;
    int heads, d, page, pages, bpp;  // bpp: blocks of a page
    int batch, cols, tokens, max_tokens;
    FastDiv by_heads, by_bpp, by_most, by_chunks, by_eighths;  // (set by the launchers) most blocks of a sequence, 16 and 8 dims
    KvTokens K, V;    // write: sources
    void *outk, *outv;  // read: destinations
};

cudaError_t launch_kv_write(const KvCacheArgs &a, int dtype, cudaStream_t st);
cudaError_t launch_kv_read(const KvCacheArgs &a, int dtype, cudaStream_t st);
// (4-bit: k points at the blocks, v and scales are not used)
cudaError_t launch_kv4_write(const KvCacheArgs &a, int dtype, cudaStream_t st);
cudaError_t launch_kv4_read(const KvCacheArgs &a, int dtype, cudaStream_t st);

// Rotary positions: one or two tensors of rows
struct RotaryPart {
    const void *x;
    void *y;
    int64_t x_token, x_head, y_token, y_head;
    int heads;
};
struct RotaryArgs {
    const int32_t *pos, *cu;
    const uint64_t *turns;
    int batch, tokens, max_tokens, dims, interleaved;
    int copied;         // dims behind the rotated ones that a call with other outputs copies
    int heads;          // of the part with more
    float gain, sine;   // factors of cosine and sine: the sine's is negative for a transposed call
    RotaryPart part[2];
    int tile, cuts;     // (set by the launcher) tokens of a CTA, CTAs that share a token's heads
    FastDiv by_half, by_units;
};
// vec: elements of a vector that all rows are aligned to
cudaError_t launch_rotary(const RotaryArgs &a, int dtype, int vec, cudaStream_t st);

struct KvAttnArgs {
    const uint8_t *k, *v;
    const float2 *scales;
    const int32_t *table, *pos, *cu;
    int heads, d, page, pages, bpp, cols, tokens, max_tokens;
    int b0, nb;  // sequences of this launch
    int group, causal, window, dtype;
    FastDiv by_heads, by_group, by_bpp;
    float scale_log2;
    const void *Q;
    int64_t q_token, q_head;
    int q_wide;  // 8-byte (f32: 16-byte) vectors of Q are aligned
    void *out;
    float *lse;
    int32_t *status;
    float most;        // largest magnitude of an f16 output (skm_kv.cu)
    float *part_cta;   // [grid][2] partial rows of units that CTAs share
    float *part_warp;  // [grid][warps] rows of the unit that a warp found begun and left
    int max_tiles;     // row tiles of the longest sequence
    int whole;         // one CTA a unit (a sequence's row tile and head)
    unsigned long long wait_ns;  // skm_kv_rows.cuh, k_kv4_prompt.cu: limit of a wait
    int stuck;         // (SKM_FAULT_WAIT) the warp whose first keys never count as arrived, k_kv4_prompt.cu: the CTA and its first or second
                       // tile of keys, 2 CTA + tile; -1: none
};
constexpr unsigned long long KV_WAIT_NS = 2000000000ull, KV_WAIT_NS_INJECTED = 1000000ull;

// How one call is run: rows a tile holds, warps, ring stages, sequences of a launch, CTAs, workspace.
struct KvRowsPlan {
    int fp32, rt, nw, ns, whole, seqs;
    int64_t units, grid;
    size_t smem, part_cta, part_warp;  // bytes
};
KvRowsPlan kv_rows_plan(int nb, int heads, int group, int d, int dtype, int max_tokens, int64_t span);
// workspace of any call of these sizes or smaller ones at most
size_t kv_rows_part_most(int nb, int heads, int d, int dtype, int64_t rows, int64_t span);
cudaError_t launch_kv_rows(const KvAttnArgs &a, const KvRowsPlan &p, cudaStream_t st);
KvRowsPlan kv4_rows_plan(int nb, int heads, int group, int d, int dtype, int max_tokens, int64_t span);
size_t kv4_rows_part_most(int nb, int heads, int d, int dtype, int64_t rows, int64_t span);
cudaError_t launch_kv4_rows(const KvAttnArgs &a, const KvRowsPlan &p, cudaStream_t st);

// Many rows on tcgen05 (k_kv_prompt.cu): max_tiles in units of a CTA's rows
struct KvPromptPlan {
    int max_tiles, splits;
    int64_t units;
    size_t part;  // bytes
};
// 16-bit rows that are always the few-row kernels'.  (Over the 4-bit cache, up to 128 dims, 20 rows of 128 units that see 5000 keys take 66 us
// there and 58 in the kernel for many rows, of 2 units 23 and 18; f16 92 and 172, 26 and 27; 12 rows, bf16, 44 and 58, 15.6 and 18)
constexpr int KV_ROWS_MOST = 32;
bool kv_prompt_ok(int dtype, int nb, int heads, int d, int64_t rows, int64_t span);
KvPromptPlan kv_prompt_plan(int nb, int heads, int group, int d, int max_tokens, int64_t span);
// workspace of any call of this d and span at most
size_t kv_prompt_part_most(int d, int64_t span);
cudaError_t launch_kv_prompt(const KvAttnArgs &a, const KvPromptPlan &p, cudaStream_t st);
// (4-bit: chosen and planned by the 8-bit cache's functions; both kernels assert the rows of a CTA that they count on)
cudaError_t launch_kv4_prompt(const KvAttnArgs &a, const KvPromptPlan &p, cudaStream_t st);

// A kernel's shared-memory limit, raised once a device: the call costs a
// microsecond, as much as a fifth of a small launch.  A launch that is refused (the
// device was reset since) raises it again.
struct SmemLimit {
    std::atomic<uint64_t> raised{0};
    template <class Kernel, class Launch>
    cudaError_t launch(Kernel *kern, size_t bytes, Launch &&go) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = uint64_t(1) << (dev & 63);
        for (int again = 0;; ++again) {
            const bool was = dev < 64 && (raised.load(std::memory_order_relaxed) & bit) && !again;
            if (!was) {
                e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
                if (e != cudaSuccess) return e;
                raised.fetch_or(bit, std::memory_order_relaxed);
            }
            go();
            if (!was || cudaPeekAtLastError() != cudaErrorInvalidValue) return launched();
            cudaGetLastError();
        }
    }
};

// ---- device helpers
__device__ __forceinline__ float kv_code(uint32_t word, int byte) {
    // 2^23 + u as a float's bits, minus 2^23 + 128
    return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440 | byte)) - 8388736.0f;
}
__device__ __forceinline__ float kv_load(const void *x, int64_t i, int dtype) {
    if (dtype == SKM_DTYPE_F32) return static_cast<const float *>(x)[i];
    if (dtype == SKM_DTYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(x)[i]);
    return __half2float(static_cast<const __half *>(x)[i]);
}
__device__ __forceinline__ void kv_store(void *x, int64_t i, float v, int dtype) {
    if (dtype == SKM_DTYPE_F32) static_cast<float *>(x)[i] = v;
    else if (dtype == SKM_DTYPE_BF16) static_cast<__nv_bfloat16 *>(x)[i] = __float2bfloat16_rn(v);
    else static_cast<__half *>(x)[i] = __float2half_rn(v);
}
// two f16, beyond f16's largest numbers those; NaN stays
__device__ __forceinline__ uint32_t kv_f16_within(float a, float b) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
// brought into [-most, most]; NaN stays
__device__ __forceinline__ float kv_within(float x, float most) { return x > most ? most : x < -most ? -most : x; }
// two fp32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\t"
        "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmov.b64 rc, {%6, %7};\n\t"
        "fma.rn.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 ra, rb, rd;\n\t"
        "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
        "add.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 ra, rb, rd;\n\t"
        "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
        "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ int kv_clamp(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// the rows [x, x + y) of sequence b in the token tensors
__device__ __forceinline__ int2 kv_rows_of(const int32_t *cu, int b, int tokens, int most) {
    const int c0 = kv_clamp(cu[b], 0, tokens), c1 = kv_clamp(cu[b + 1], c0, tokens);
    return make_int2(c0, min(c1 - c0, most));
}

}  // namespace skm
