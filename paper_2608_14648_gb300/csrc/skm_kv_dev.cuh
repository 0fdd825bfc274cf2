// Device helpers of the attention kernels over the 8-bit cache (k_kv_rows.cu,
// k_kv_prompt.cu) and the 4-bit one (k_kv4_rows.cu, k_kv4_prompt.cu).
#pragma once
#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr float M_NONE = -3.0e38f;  // the reference before the first logit
constexpr float M_SLACK = 15.0f, M_BELOW = 7.0f, M_MOST = 32768.0f;  // M_MOST = 2^M_SLACK
constexpr float LN2 = 0.69314718055994531f;

__device__ __forceinline__ float ex2(float x) {  // 2^x, 2 units in the last place, subnormal results 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t su32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool bar_try(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(ok)
        : "r"(b), "r"(parity)
        : "memory");
    return ok != 0;
}
// false after `limit` ns
__device__ __forceinline__ bool bar_wait(uint32_t b, uint32_t parity, unsigned long long limit) {
    if (bar_try(b, parity)) return true;
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (uint32_t i = 1;; ++i) {
        if (bar_try(b, parity)) return true;
        if ((i & 63) == 0) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t - t0 > limit) return false;
        }
    }
}
__device__ __forceinline__ void bulk_g2s(uint32_t dst, const void *src, uint32_t bytes, uint32_t b) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
        "l"(src), "r"(bytes), "r"(b)
        : "memory");
}

// ---- a sequence as this launch sees it
struct Seq {
    int lo, cnt;  // first block (of T tokens) that a row sees, blocks
    int len, n;   // tokens held, rows
    int row0;     // its first row in the token tensors
};
template <int T = KV_B>
__device__ __forceinline__ Seq seq_of(const KvAttnArgs &a, int b) {
    Seq s;
    s.len = kv_clamp(a.pos[b], 0, a.cols * a.page);
    const int2 rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
    s.row0 = rows.x;
    s.n = rows.y;
    s.lo = a.window > 0 ? max(0, s.len - s.n - a.window + 1) / T : 0;
    s.cnt = s.n > 0 ? (s.len + T - 1) / T - s.lo : 0;
    if (s.cnt < 0) s.cnt = 0;
    return s;
}
__device__ __forceinline__ int tiles_of(const KvAttnArgs &a, const Seq &s, int rt) {
    return (int)(((int64_t)s.n * a.group + rt - 1) / rt);
}
// the last / first position that row r of a sequence may see (last < first: none)
__device__ __forceinline__ int last_of(const KvAttnArgs &a, const Seq &s, int r) {
    const int i = a.by_group.div(r);
    if (i >= s.n) return -1;
    return a.causal ? min(s.len - 1, s.len - s.n + i) : s.len - 1;
}
__device__ __forceinline__ int first_of(const KvAttnArgs &a, const Seq &s, int r) {
    return a.window > 0 ? max(0, s.len - s.n + a.by_group.div(r) - a.window + 1) : 0;
}

// Where a row's result goes
__device__ __forceinline__ int64_t row_index(const KvAttnArgs &a, const Seq &s, int h, int r) {
    return ((int64_t)s.row0 + a.by_group.div(r)) * (a.heads * a.group) + h * a.group + a.by_group.mod(r);
}

// A block's scales as attention uses them: (key scale, log2 of the value scale,
// 1 / value scale, 0).  Weights carry the value scale, so scales too far apart would push
// the smaller ones' weights out of fp32: scales below 2^-80 (values below 1e-22,
// blocks of zeros among them) count as 2^-80.  (The reference lies at least 7 below the row's largest
// weight, so that one is 2^7 or more; fp32 ends at 2^-126, and weights down to 2^-24 of the largest count
// in a row's sum: scales may lie 2^(126 + 7 - 24) = 2^109 apart.)
__device__ __forceinline__ float4 value_scale(float2 sc) {
    const float vs = fmaxf(sc.y, 8.271806e-25f);
    float lg, inv;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lg) : "f"(vs));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(vs));
    return make_float4(sc.x, lg, inv, 0.0f);
}

// A bf16 query row becomes f16 by a power of two that takes its largest element to [2^15, 2^16) (65280 at
// most, of f16's 65504; the products of 256 dims with codes stay below 2^32).  That is exact for elements of 2^-32 of the
// largest and more: the eight bits of one lie above 2^-24, f16's smallest number.  ex: the largest
// element's exponent field
struct Pow2 {
    float mul, back;
};
__device__ __forceinline__ Pow2 to_f16(uint32_t ex, uint32_t most = 15u) {
    const uint32_t e = max(ex, 1u), up = min(e - 1u, most);
    return Pow2{__uint_as_float((254u - e + up) << 23), __uint_as_float((e - up) << 23)};
}

// codes of bytes 0, 1 / 2, 3 of a word as two f16: 1024 + u as bits, minus 1152
__device__ __forceinline__ uint32_t codes_f16(uint32_t word, uint32_t sel) {
    const uint32_t x = __byte_perm(word, 0x64646464u, sel);
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&x), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t *>(&r);
}
}  // namespace

}  // namespace skm
