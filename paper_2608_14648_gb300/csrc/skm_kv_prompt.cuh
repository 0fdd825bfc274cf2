// Attention over a key/value cache for many query rows on tcgen05: what the 8-bit
// cache's kernel (k_kv_prompt.cu) and the 4-bit cache's (k_kv4_prompt.cu) share: barriers, products, TMEM,
// query rows as an operand, the kernel that joins parts.
#pragma once
#include <type_traits>

#include "skm_kv_dev.cuh"

namespace skm {

namespace {

constexpr int QT = 128, KT = 64, KBLK = KT / KV_B;  // rows of a tile, keys of a tile, blocks of it
constexpr int RANKED = 256;
// rows of a CTA: two row tiles, above 128 dims one.  Units, parts and workspaces of both caches' kernels are planned with it
// (kv_prompt_plan, kv_prompt_part_most)
__host__ __device__ constexpr int prompt_rows(int d) { return d <= 128 ? 2 * QT : QT; }

__device__ __forceinline__ void arrive(uint32_t b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory");
}
// bounded, and cut short when another role gave up
__device__ __forceinline__ bool wait(uint32_t b, uint32_t parity, volatile int32_t *gone) {
    if (bar_try(b, parity)) return true;
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (uint32_t i = 1;; ++i) {
        if (bar_try(b, parity)) return true;
        if ((i & 63) == 0) {
            if (*gone) return false;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t - t0 > KV_WAIT_NS) {
                *gone = 1;
                return false;
            }
        }
    }
}
// by a whole warp, with one answer
__device__ __forceinline__ bool warp_wait(uint32_t b, uint32_t parity, volatile int32_t *gone) {
    return __all_sync(0xffffffffu, wait(b, parity, gone));
}
// whether a phase is over, without the wait that a try may include
__device__ __forceinline__ bool bar_test(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(ok)
        : "r"(b), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// The issuing warp runs its loop converged and one elected lane (`one`) takes the
// tcgen05 instructions by predicate, not by a branch: the operands then stay in
// uniform registers.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void commit(uint32_t b, uint32_t one) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(b),
        "r"(one)
        : "memory");
}
// K-major operand, 128-byte swizzle: rows of 128 bytes, groups of 8 rows
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
constexpr uint32_t idesc(int n) {  // f16 x f16 -> f32, M = 128, both K-major
    return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(QT >> 4) << 24);
}
template <bool ADD>
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t one) {
    asm volatile(
        "{\n\t.reg .pred e, p;\n\tsetp.ne.b32 e, %4, 0;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"(one), "n"(ADD)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t add, uint32_t one) {
    asm volatile(
        "{\n\t.reg .pred e, p;\n\tsetp.ne.b32 e, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(id), "r"(add), "r"(one)
        : "memory");
}
// 16 columns; valid after ld_wait on the same registers
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void ld_wait(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]),
                   "+r"(v[15])
                 :
                 : "memory");
}
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_shared(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// two weights 2^a, 2^b as f16, and added to a pair of sums (the sums as 64 bits, the
// weights' conversion from the pair that was added: fewer moves between registers)
__device__ __forceinline__ uint32_t weights2(float a, float b, uint64_t &sum) {
    uint32_t p;
    asm("{\n\t.reg .b64 e;\n\t.reg .f32 x, y;\n\t"
        "ex2.approx.ftz.f32 x, %2;\n\tex2.approx.ftz.f32 y, %3;\n\t"
        "mov.b64 e, {x, y};\n\tadd.rn.f32x2 %1, %1, e;\n\t"
        "mov.b64 {x, y}, e;\n\tcvt.rn.f16x2.f32 %0, y, x;\n\t}"
        : "=r"(p), "+l"(sum)
        : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float2 halves(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}

__device__ __forceinline__ uint64_t joined(float2 x) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x.x), "f"(x.y));
    return r;
}

// A part: a CTA's rows x (m, l), then its rows of d sums
__host__ __device__ __forceinline__ int64_t prompt_part(int rows, int d) { return rows * (int64_t)(2 + d); }

// 8 values without the alignment of a vector (not inlined: a rare path)
__device__ __noinline__ uint4 load8(const uint16_t *x) {
    uint32_t w[4];
    for (int i = 0; i < 4; ++i) w[i] = x[2 * i] | (uint32_t)x[2 * i + 1] << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint32_t bf16_f16(uint32_t w, float mul) {
    return pack(__uint_as_float(w << 16) * mul, __uint_as_float(w & 0xffff0000u) * mul);
}

// A warp's 32 query rows to f16 in their tile's operand, DH / 8 lanes a row, all
// reads issued before the first is used; returns what the logits of row `lane` are
// multiplied by (bf16 rows are scaled by a power of two: to_f16).  tile0: the
// tile's row 0, row0: the warp's first row of it.  Infinities and NaN enter as zeros (with their neighbours)
// and are noted in `wild`, a byte a row of the tile: such a row becomes NaN at the end if it has seen a key.  (An
// absent block's keys are zeros here: their products would be NaN where the row sees nothing.)
// UP: the largest element's exponent, both types scaled (15 or less; F16 rows as they are where it is 15).  SUM: row `lane`'s sum as the
// operand has it.
template <int DH, bool SUM = false, uint32_t UP = 15>
__device__ __forceinline__ float load_rows(const KvAttnArgs &a, const Seq &s, int h, int tile0, int row0, uint32_t tile, int lane,
                                            uint8_t *wild, float *sum = nullptr) {
    constexpr int LPR = DH / 8, RPI = 32 / LPR, IT = 32 / RPI, AT_ONCE = IT < 16 ? IT : 16;
    const int li = lane % LPR, sub = lane / LPR;
    float fac = a.scale_log2;
    wild[row0 + lane] = 0;
    __syncwarp();
    for (int i0 = 0; i0 < IT; i0 += AT_ONCE) {
        uint4 raw[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = tile0 + row0 + (i0 + i) * RPI + sub;
            raw[i] = make_uint4(0, 0, 0, 0);
            if (r < s.n * a.group && 8 * li < a.d) {
                const int t = a.by_group.div(r);
                const uint16_t *x = static_cast<const uint16_t *>(a.Q) + (int64_t)(s.row0 + t) * a.q_token +
                                    (int64_t)(h * a.group + r - t * a.group) * a.q_head + 8 * li;
                if (a.q_wide) {
                    const uint2 u = *reinterpret_cast<const uint2 *>(x), v = *reinterpret_cast<const uint2 *>(x + 4);
                    raw[i] = make_uint4(u.x, u.y, v.x, v.y);
                } else {
                    raw[i] = load8(x);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int row = row0 + (i0 + i) * RPI + sub;
            uint4 w = raw[i];
            if (UP < 15 && a.dtype != SKM_DTYPE_BF16) {
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                float2 y[4];
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    y[k] = __half22float2(*reinterpret_cast<const __half2 *>(u + k));
                    top = max(max(top, __float_as_uint(y[k].x) & 0x7fffffffu), __float_as_uint(y[k].y) & 0x7fffffffu);
                }
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const Pow2 by = to_f16(top >> 23, UP);
                if (top >= 0x7f800000u) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = make_float2(0.0f, 0.0f);
                    wild[row] = 1;
                }
                w = make_uint4(pack(y[0].x * by.mul, y[0].y * by.mul), pack(y[1].x * by.mul, y[1].y * by.mul), pack(y[2].x * by.mul, y[2].y * by.mul),
                               pack(y[3].x * by.mul, y[3].y * by.mul));
                const float mine = __shfl_sync(0xffffffffu, by.back, (lane % RPI) * LPR);
                if (lane / RPI == i0 + i) fac = mine * a.scale_log2;
            } else if (a.dtype == SKM_DTYPE_BF16) {
                uint32_t top = 0;  // the largest |x| as bits
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) top = max(max(top, u[k] << 16 & 0x7fff0000u), u[k] & 0x7fff0000u);
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const Pow2 by = to_f16(top >> 23, UP);
                if (top >= 0x7f800000u) {
                    w = make_uint4(0, 0, 0, 0);
                    wild[row] = 1;
                }
                w = make_uint4(bf16_f16(w.x, by.mul), bf16_f16(w.y, by.mul), bf16_f16(w.z, by.mul), bf16_f16(w.w, by.mul));
                const float mine = __shfl_sync(0xffffffffu, by.back, (lane % RPI) * LPR);
                if (lane / RPI == i0 + i) fac = mine * a.scale_log2;
            } else {  // (an exponent of ones carries into the sign's place)
                const auto ends = [](uint32_t x) { return (x & 0x7c007c00u) + 0x04000400u; };
                if ((ends(w.x) | ends(w.y) | ends(w.z) | ends(w.w)) & 0x80008000u) {
                    w = make_uint4(0, 0, 0, 0);
                    wild[row] = 1;
                }
            }
            if constexpr (SUM) {
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                float x = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(u + k));
                    x += y.x + y.y;
                }
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
                x = __shfl_sync(0xffffffffu, x, (lane % RPI) * LPR);
                if (lane / RPI == i0 + i) *sum = x;
            }
            st_shared(tile + (li >> 3) * (QT * 128) + row * 128 + (((li & 7) ^ (row & 7)) << 4), w.x, w.y, w.z, w.w);
        }
    }
    return fac;
}

// A CTA takes 8 rows of a unit; the threads of a row its dims.
__global__ void __launch_bounds__(256) kv_prompt_join_kernel(const __grid_constant__ KvAttnArgs a, int splits, int unit_rows,
                                                             const float *parts) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tiles = a.max_tiles;
    const int unit = blockIdx.x / (unit_rows / 8), pr = blockIdx.x % (unit_rows / 8) * 8 + (threadIdx.x >> 5);
    const int h = a.by_heads.mod(unit), u = a.by_heads.div(unit);
    const int b = a.b0 + u / tiles, r = u % tiles * unit_rows + pr;
    const Seq s = seq_of(a, b);
    if (r >= s.n * a.group) return;
    const float *base = parts + (int64_t)unit * splits * prompt_part(unit_rows, a.d);
    float m = M_NONE, l = 0.0f;
    for (int i = 0; i < splits; ++i) m = fmaxf(m, base[i * prompt_part(unit_rows, a.d) + 2 * pr]);
    const int64_t row = row_index(a, s, h, r);
    for (int i = 0; i < splits; ++i) {
        const float *p = base + i * prompt_part(unit_rows, a.d) + 2 * pr;
        l = fmaf(p[1], exp2f(p[0] - m), l);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    for (int c = threadIdx.x & 31; c < a.d / 4; c += 32) {
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int i = 0; i < splits; ++i) {
            const float *p = base + i * prompt_part(unit_rows, a.d);
            const float w = exp2f(p[2 * pr] - m);
            const float4 v = *reinterpret_cast<const float4 *>(p + 2 * unit_rows + (int64_t)pr * a.d + 4 * c);
            o.x = fmaf(v.x, w, o.x), o.y = fmaf(v.y, w, o.y), o.z = fmaf(v.z, w, o.z), o.w = fmaf(v.w, w, o.w);
        }
        const float most = a.dtype == SKM_DTYPE_F16 ? a.most : INFINITY;
        kv_store(a.out, row * a.d + 4 * c, kv_within(o.x * inv, most), a.dtype);
        kv_store(a.out, row * a.d + 4 * c + 1, kv_within(o.y * inv, most), a.dtype);
        kv_store(a.out, row * a.d + 4 * c + 2, kv_within(o.z * inv, most), a.dtype);
        kv_store(a.out, row * a.d + 4 * c + 3, kv_within(o.w * inv, most), a.dtype);
    }
    if ((threadIdx.x & 31) == 0 && a.lse) a.lse[row] = l == 0.0f ? -INFINITY : LN2 * (m + log2f(l));
}

cudaError_t run_prompt_join(const KvAttnArgs &a, const KvPromptPlan &p, int unit_rows, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.units * (unit_rows / 8)));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_prompt_join_kernel, a, p.splits, unit_rows, (const float *)a.part_cta);
    return e != cudaSuccess ? e : launched();
}

}  // namespace

}  // namespace skm
