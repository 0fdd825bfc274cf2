// Attention over the 8-bit cache for many query rows (prompt chunks) on
// tcgen05: 16-bit queries.
//
// A CTA takes 256 query rows (token-major, then the heads of a group) of one
// sequence and key/value head as two tiles of 128 (d > 128: one tile, so that its
// sums fit TMEM and its operands shared memory), and walks the keys they see in
// tiles of 64 positions (4 blocks of the cache).  The codes are exact in f16, so
// both products run in kind::f16 and the block scales stay out of the
// operands: the key scale multiplies the logits of its block, the value scale
// is added to them as log2 s_v (o = sum p c_v, l = sum p / s_v; the formulas of
// k_kv_rows.cu, the running reference m included).
//
//   warps 0-3, 4-7  softmax of tile 0 / 1, one thread a row: 16 logits at a time
//                   from TMEM, the next 16 already on their way, p = 2^(s f + c) to
//                   f16, P back to TMEM over the columns S held (the A operand of
//                   the next product)
//   warps 8-14      converters: a block of keys (or values) at a time from
//                   global memory, one block ahead in registers, to f16 in the
//                   128-byte-swizzled operand layout
//   warp 15         MMA issuer (d > 128: 4 softmax warps, the others behind them)
//
// TMEM: two S/P buffers of 64 columns a tile, O0, O1 (DH columns each).  The
// logits of a key tile are under way while the softmax of the one before runs (with one buffer
// of 128 keys a tile the chain softmax, P V, Q K' took 5400 clocks for 256 x 128
// logits where the tensor cores need 2048).  The pass over a tile's
// logits assumes that m need not move; the first tile, and a block whose sum exceeds
// 65000 (seldom), send the warp through the maxima, a rescaling of O and the weights
// once more.  Shared memory: Q, and rings of K and V tiles.
//
// Few CTAs (short prompts): the keys are split over CTAs as well, and
// kv_prompt_join_kernel merges the parts in order.
//
// Measured (GB300): chunks of 2048 tokens of two prompts behind 6144, 32 query heads
// over 8 of 128, bf16: 298 us = 1130 TFLOP/s, 59% of a cuBLAS product; 4 whole prompts of up to
// 4096, 16 heads of 64, f16: 124 us (half the flops a logit, and key tiles on the
// diagonal).  A tile of 256 rows x 64 keys takes some 2000 clocks.  What bounds it is the
// softmax warps' chain of latencies, two warps a scheduler: in copies of 290 us, without the
// exponentials, the conversion of codes or P's way back the time stays within 2%, with three
// quarters of the products gone it is 276 us, without exponentials and conversion as well
// 248.  The loops are at the limit of 128 registers, and a few instructions outside them move the time by 2%:
// noting query rows with infinities or NaN costs 5 us.  So reads
// that a wait would hold up come before it (a block's scales: 11 us), the converters
// leave issue slots free (6 us), and what runs seldom stays in its branch.  More logits a
// wait (367 us) or asking for the next tile's earlier (311) made it slower.
#include "skm_kv_dev.cuh"

namespace skm {

namespace {

constexpr int QT = 128, KT = 64, KBLK = KT / KV_B;  // rows of a tile, keys of a tile, blocks of it
constexpr int CONV = 7;  // converter warps
constexpr int RANKED = 256;
constexpr float W_MOST = 65000.0f;  // a block's sum of weights: above it one may pass the largest f16
// tiles whose scales are kept.  A K stage is free once its product is through, which is issued when the softmax has
// handed over the tile two before: tile j + ST (at most 4) comes while it reads tile j - 1 at the earliest, 5 behind
constexpr int INFO = 8;

// DH: dims, padded to 64, 128 or 256
template <int DH>
struct Lay {
    static constexpr int NQ = DH <= 128 ? 2 : 1;      // row tiles of a CTA
    static constexpr int ST = DH <= 128 ? 4 : 2;      // K and V tiles in flight
    static constexpr int ROWS = NQ * QT;
    static constexpr int CONV_WARP0 = 4 * NQ, MMA_WARP = CONV_WARP0 + CONV, THREADS = 32 * (MMA_WARP + 1);
    static constexpr int QTILE = QT * DH * 2, TILE = KT * DH * 2;  // bytes of a Q tile, of a K or V tile
    static constexpr int q = 0, k = NQ * QTILE, v = k + ST * TILE, info = v + ST * TILE;
    static constexpr int bars = info + INFO * KBLK * 16, slots = bars + 8 * (4 * ST + 14);  // TMEM address, a flag, the part's index
    static constexpr int wild = slots + 32;  // a byte a row: its query holds infinities or NaN
    // one CTA an SM: it takes all of TMEM
    static constexpr int bytes = wild + ROWS + 1024, total = bytes > 120 * 1024 ? bytes : 120 * 1024;
    static constexpr uint32_t O = NQ * 2 * KT;  // TMEM column of O0
};

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
template <int DH>
__device__ __forceinline__ float load_rows(const KvAttnArgs &a, const Seq &s, int h, int tile0, int row0, uint32_t tile, int lane,
                                            uint8_t *wild) {
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
            if (a.dtype == SKM_DTYPE_BF16) {
                uint32_t top = 0;  // the largest |x| as bits
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) top = max(max(top, u[k] << 16 & 0x7fff0000u), u[k] & 0x7fff0000u);
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const Pow2 by = to_f16(top >> 23);
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
            st_shared(tile + (li >> 3) * (QT * 128) + row * 128 + (((li & 7) ^ (row & 7)) << 4), w.x, w.y, w.z, w.w);
        }
    }
    return fac;
}

template <int DH>
__global__ void __launch_bounds__(Lay<DH>::THREADS, 1)
    kv_prompt_kernel(const __grid_constant__ KvAttnArgs a, int splits, float *parts) {
    using L = Lay<DH>;
    constexpr int ST = L::ST, ROWS = L::ROWS, CONV_WARP0 = L::CONV_WARP0, MMA_WARP = L::MMA_WARP, THREADS = L::THREADS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t *smem = smem_raw + ((1024 - (su32(smem_raw) & 1023)) & 1023);  // swizzle atoms
    const uint32_t sm = su32(smem);
    const auto bar = [&](int i) { return sm + L::bars + 8 * i; };
    const auto k_full = [&](int s) { return bar(s); };
    const auto k_free = [&](int s) { return bar(ST + s); };
    const auto v_full = [&](int s) { return bar(2 * ST + s); };
    const auto v_free = [&](int s) { return bar(3 * ST + s); };
    const auto s_full = [&](int q, int buf) { return bar(4 * ST + 2 * q + buf); };
    const auto p_full = [&](int q, int buf) { return bar(4 * ST + 4 + 2 * q + buf); };
    const auto o_done = [&](int q) { return bar(4 * ST + 8 + q); };
    const auto o_last = [&](int q) { return bar(4 * ST + 10 + q); };
    const uint32_t q_full = bar(4 * ST + 12), drain = bar(4 * ST + 13);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::slots);
    volatile int32_t *gone = reinterpret_cast<volatile int32_t *>(smem + L::slots + 4);
    float4 *info = reinterpret_cast<float4 *>(smem + L::info);  // a block's value_scale, its log2 -infinity where the block is absent

    // the unit: ROWS rows of a sequence, longest first where there is more than one a
    // SM (few units are ranked by the key tiles they see; of many, the later rows come first), its heads next
    // to each other
    const int tiles = a.max_tiles, pairs = a.nb * tiles;
    int u = blockIdx.x;
    const int split = u % splits;
    u /= splits;
    const int h = a.by_heads.mod(u);
    u = a.by_heads.div(u);
    if (pairs <= RANKED && gridDim.x > KV_SMS) {
        int *length = reinterpret_cast<int *>(smem), *pick = length + RANKED;
        if (tid < pairs) {
            const Seq s = seq_of(a, a.b0 + tid / tiles);
            const int r0 = tid % tiles * ROWS, r1 = min(r0 + ROWS, s.n * a.group) - 1;
            length[tid] = r1 < r0 ? -1 : last_of(a, s, r1) / KT - first_of(a, s, r0) / KT;
        }
        __syncthreads();
        if (tid < pairs) {
            int rank = 0;
            for (int i = 0; i < pairs; ++i) rank += length[i] > length[tid] || (length[i] == length[tid] && i < tid);
            if (rank == u) *pick = tid;
        }
        __syncthreads();
        u = *pick;
        __syncthreads();
    } else {
        u = u % a.nb * tiles + tiles - 1 - u / a.nb;
    }
    const int bi = u / tiles, pair = u % tiles, b = a.b0 + bi;
    int64_t *part_index = reinterpret_cast<int64_t *>(smem + L::slots + 8);
    if (tid == 0) *part_index = ((int64_t)u * a.heads + h) * splits + split;
    const Seq s = seq_of(a, b);
    const int rows = s.n * a.group, r0 = pair * ROWS;
    if (r0 >= rows) return;
    const int r1 = min(r0 + ROWS, rows) - 1;
    const int nq = r1 - r0 >= QT ? 2 : 1;
    // positions that some row sees, the tiles of them, this split's tiles
    const int first = first_of(a, s, r0), last = last_of(a, s, r1);
    const int t_lo = first / KT, t_all = last >= first ? last / KT + 1 - t_lo : 0;
    const int t0 = t_lo + (int)((int64_t)t_all * split / splits);
    const int n = t_lo + (int)((int64_t)t_all * (split + 1) / splits) - t0;
    // those that a row tile goes through: the last one all of them, the one before it to its own end
    const auto tiles_for = [&](int q) {
        if (q >= nq) return 0;
        const int its_last = last_of(a, s, min(r0 + (q + 1) * QT - 1, r1));
        return its_last < first ? 0 : kv_clamp(its_last / KT + 1 - t0, 0, n);
    };

    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(k_full(i)), "r"(KBLK) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(v_full(i)), "r"(KBLK) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(k_free(i)), "r"(1) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(v_free(i)), "r"(1) : "memory");
        }
        for (int q = 0; q < L::NQ; ++q) {
            for (int i = 0; i < 2; ++i) {
                asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(s_full(q, i)), "r"(1) : "memory");
                asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(p_full(q, i)), "r"(4) : "memory");
            }
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(o_done(q)), "r"(1) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(o_last(q)), "r"(1) : "memory");
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(q_full), "r"(4 * L::NQ) : "memory");
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(drain), "r"(1) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *gone = 0;
    }
    if (a.d < DH) {  // dims from d on are zeros
        for (int i = tid * 16; i < 2 * ST * L::TILE; i += THREADS * 16) st_shared(sm + L::k + i, 0, 0, 0, 0);
        fence_async();
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(tmem_slot)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp < CONV_WARP0) {  // ------------------------------------------ softmax
        const int q = warp >> 2, row = (warp & 3) * 32 + lane, r = r0 + q * QT + row, nt = tiles_for(q);
        const bool in = r < rows;
        const float fac = load_rows<DH>(a, s, h, r0 + q * QT, (warp & 3) * 32, sm + L::q + q * L::QTILE, lane,
                                        smem + L::wild + q * QT);
        fence_async();
        __syncwarp();
        if (lane == 0) arrive(q_full);
        // (rows past the end see everything, with no weight: they slow no one down)
        const int hi = in ? last_of(a, s, r) : 0x7ffffffe, lo = in ? first_of(a, s, r) : 0;
        // rows of the warp see [low, high] whole
        const int high = __shfl_sync(0xffffffffu, hi, 0), low = __reduce_max_sync(0xffffffffu, lo);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S0 = tmem + lanes + q * 2 * KT, O = tmem + lanes + L::O + q * DH;
        float m = in ? M_NONE : -M_NONE, l = 0.0f;
        bool ok = true, loaded = false;  // loaded: v[0] holds (or will) the first logits of tile j
        uint32_t v[2][16];
        for (int j = 0; j < nt; ++j) {
            const uint32_t S = S0 + (j & 1) * KT;
            if (!loaded) {
                if (!(ok = warp_wait(s_full(q, j & 1), (j >> 1) & 1, gone))) break;
                fence_after();
                if (j > 0) ld16(S, v[0]);
            }
            const float4 *inf = info + (j & (INFO - 1)) * KBLK;
            const int c0 = (t0 + j) * KT;
            const bool whole = c0 >= low && c0 + KT - 1 <= high;
            uint32_t P[KT / 2];
            float most = 0.0f, add = 0.0f;
            // the positions of block k that the row sees, as bits (opaque, so that it stays in the
            // branches that ask: hoisted, it ran in every tile)
            const auto visible = [&](int k) {
                int at = c0 + k * KV_B;
                asm volatile("" : "+r"(at));
                return ((1u << kv_clamp(hi + 1 - at, 0, KV_B)) - 1) & ~0u << kv_clamp(lo - at, 0, KV_B);
            };
            // weights of block k of the tile from 16 logits
            const auto weigh = [&](const uint32_t (&x)[16], int k, float4 f4) {
                const float f = fac * f4.x, c = f4.y - m;
                float p[16];
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float2 t = fma2(make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), make_float2(f, f),
                                          make_float2(c, c));
                    p[i] = t.x, p[i + 1] = t.y;
                }
                if (!whole) {
                    const uint32_t sees = visible(k);
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[i] = sees & 1u << i ? p[i] : -INFINITY;
                }
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 16; i += 2) P[k * 8 + i / 2] = weights2(p[i], p[i + 1], sum[(i >> 1) & 1]);
                const float2 both = halves(add2(sum[0], sum[1]));
                const float all = both.x + both.y;
                most = fmaxf(most, all);
                add = fmaf(all, f4.z, add);
            };
            bool moves = j == 0;  // the reference: set by the first tile, seldom moved by a later one
            if (!moves) {
                float4 coming;
#pragma unroll
                for (int k = 0; k < KBLK; ++k) {
                    const float4 now = k ? coming : inf[0];
                    if (k + 1 < KBLK) coming = inf[k + 1];  // (read before the wait, which nothing moves across)
                    ld_wait(v[k & 1]);
                    if (k + 1 < KBLK) {
                        ld16(S + (k + 1) * KV_B, v[(k + 1) & 1]);
                    } else {  // the next tile's first logits, if they are there
                        loaded = j + 1 < nt && __all_sync(0xffffffffu, bar_test(s_full(q, (j + 1) & 1), ((j + 1) >> 1) & 1));
                        if (loaded) {
                            fence_after();
                            ld16(S0 + ((j + 1) & 1) * KT, v[0]);
                        }
                    }
                    weigh(v[k & 1], k, now);
                }
                moves = __any_sync(0xffffffffu, most > W_MOST);
            }
            if (moves) {
                // the rows' maxima, with them new references, and the weights (again)
                uint32_t w[KBLK][16];
#pragma unroll
                for (int k = 0; k < KBLK; ++k) ld16(S + k * KV_B, w[k]);
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < KBLK; ++k) {
                    ld_wait(w[k]);
                    const float4 f4 = inf[k];
                    const float f = fac * f4.x;
                    const uint32_t sees = visible(k);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (sees & 1u << i) top = fmaxf(top, fmaf(__uint_as_float(w[k][i]), f, f4.y));
                }
                const float to = top > m + 8.0f ? top - M_BELOW : m;
                const float g = ex2(m - to);
                m = to;
                l *= g;
                if (j > 0) {
                    if (!(ok = warp_wait(o_done(q), (j - 1) & 1, gone))) break;
                    fence_after();
#pragma unroll 1
                    for (int k = 0; k < DH / 16; ++k) {
                        uint32_t x[16];
                        ld16(O + k * 16, x);
                        ld_wait(x);
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * g);
                        st16(O + k * 16, x);
                    }
                    st_wait();
                }
                add = 0.0f;
#pragma unroll
                for (int k = 0; k < KBLK; ++k) weigh(w[k], k, inf[k]);
            }
            l += add;
#pragma unroll
            for (int k = 0; k < KT / 2; k += 16) st16(S + k, P + k);
            st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) arrive(p_full(q, j & 1));
        }
        if (loaded) ld_wait(v[0]);  // an early end leaves no load in flight
        if (q < nq) {
            if (ok && nt > 0) {
                ok = warp_wait(o_last(q), 0, gone);
                fence_after();
            }
            if (!ok) {
                l = NAN;
                if (lane == 0 && a.status) *a.status = 1;
            }
            if (smem[L::wild + q * QT + row] && l != 0.0f) l = NAN;
            float *part = parts ? parts + *part_index * prompt_part(ROWS, a.d) : nullptr;
            const int pr = q * QT + row;
            if (part) reinterpret_cast<float2 *>(part)[pr] = make_float2(m, l);
            const int64_t at = in ? row_index(a, s, h, r) : 0;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll 2
            for (int k = 0; k < DH / 16; ++k) {
                if (16 * k >= a.d) break;
                uint32_t v[16];
                __syncwarp();
                if (ok && nt > 0) {
                    ld16(O + k * 16, v);
                    ld_wait(v);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0;
                }
                if (!in) continue;
                if (part) {
                    float4 *dst = reinterpret_cast<float4 *>(part + 2 * ROWS + (int64_t)pr * a.d + 16 * k);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                                             __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                    continue;
                }
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x0 = __uint_as_float(v[2 * i]) * inv, x1 = __uint_as_float(v[2 * i + 1]) * inv;
                    if (a.dtype == SKM_DTYPE_BF16) {
                        const __nv_bfloat162 y = __floats2bfloat162_rn(x0, x1);
                        w[i] = *reinterpret_cast<const uint32_t *>(&y);
                    } else {
                        w[i] = pack(x0, x1);
                    }
                }
                uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.out) + at * a.d + 16 * k);
                dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
            if (in && !part && a.lse) a.lse[at] = l == 0.0f ? -INFINITY : LN2 * (m + log2f(l));
        }
    } else if (warp < MMA_WARP) {  // ------------------------------------- converters
        // tasks: per tile KBLK blocks of keys, then KBLK of values; warp w takes w, w + CONV, ...
        const int tasks = n * 2 * KBLK, cw = warp - CONV_WARP0;
        constexpr int NV = DH / 32;
        struct Ahead {  // 32 of the warp's tasks, one a lane
            int at;
            float2 sc;
        };
        const auto look = [&](int task) {
            Ahead w;
            w.at = -1;
            w.sc = make_float2(0.0f, 0.0f);
            if (task < tasks) {
                const int blk = (t0 + task / (2 * KBLK)) * KBLK + task % KBLK;
                if (blk * KV_B <= last && blk * KV_B + KV_B > first) {
                    const int pg = a.table[(int64_t)b * a.cols + a.by_bpp.div(blk)];
                    if (pg >= 0 && pg < a.pages) {
                        w.at = (pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk);
                        w.sc = a.scales[w.at];
                    }
                }
            }
            return w;
        };
        const auto load = [&](int task, int at, uint4 (&raw)[NV]) {
            const uint4 *p = reinterpret_cast<const uint4 *>((task & KBLK ? a.v : a.k) + (int64_t)at * (KV_B * a.d));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                raw[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);  // absent: zeros
                if (at >= 0 && lane + 32 * i < a.d) raw[i] = __ldg(p + lane + 32 * i);
            }
        };
        uint4 raw[NV], coming[NV];
        Ahead cur = look(cw + CONV * lane);
        int at = __shfl_sync(0xffffffffu, cur.at, 0);
        load(cw, at, raw);
        Ahead next = look(cw + CONV * (32 + lane));
        // where a lane's vector of 16 codes goes: two 16-byte chunks, the second one next
        // to the first.  Keys, vector lane + 32 k: chunk of dims lane / 16 + 2 k, token
        // lane % 16; values: dim lane + 32 k
        uint32_t to[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int w = (lane >> 4) + 2 * k;
            to[k] = (w >> 2) * (KT * 128) + (lane & 15) * 128 + (((w & 3) * 2 ^ (lane & 7)) << 4);
        }
        // a task from `raw`, the next one's codes on their way to `coming`
        const auto convert = [&](int task, int i, uint4 (&raw)[NV], uint4 (&coming)[NV]) {
            const int slot = i & 31, j = task / (2 * KBLK), st = j & (ST - 1), blk = task & (KBLK - 1);
            const bool vals = task & KBLK;
            const float2 sc = make_float2(__shfl_sync(0xffffffffu, cur.sc.x, slot), __shfl_sync(0xffffffffu, cur.sc.y, slot));
            if (slot == 31) {
                cur = next;
                next = look(task + CONV * (33 + lane));
            }
            const int at_next = __shfl_sync(0xffffffffu, cur.at, (i + 1) & 31);
            load(task + CONV, at_next, coming);
            if (!warp_wait(vals ? v_free(st) : k_free(st), ((j / ST) & 1) ^ 1, gone)) return false;
            if (!vals && lane == 0) {
                float4 f = value_scale(sc);
                if (at < 0) f.y = -INFINITY;  // an absent block: no weight (its codes are zeros)
                info[(j & (INFO - 1)) * KBLK + blk] = f;
            }
            // (a branch each for keys and values around all of it: their stores take the words in
            // other groups of four registers)
            if (!vals) {
                const uint32_t base = sm + L::k + blk * 2048 + st * L::TILE;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (lane + 32 * k >= a.d) break;
                    const uint4 c = raw[k];
                    st_shared(base + to[k], codes_f16(c.x, 0x4140), codes_f16(c.x, 0x4342), codes_f16(c.y, 0x4140),
                              codes_f16(c.y, 0x4342));
                    st_shared((base + to[k]) ^ 16, codes_f16(c.z, 0x4140), codes_f16(c.z, 0x4342), codes_f16(c.w, 0x4140),
                              codes_f16(c.w, 0x4342));
                }
            } else {  // even halves of a word tokens 0..7, odd 8..15
                const uint32_t base = sm + L::v + lane * 128 + ((blk * 2 ^ (lane & 7)) << 4) + st * L::TILE;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (lane + 32 * k >= a.d) break;
                    const uint4 c = raw[k];
                    st_shared(base + k * 4096, codes_f16(c.x, 0x4140), codes_f16(c.y, 0x4140), codes_f16(c.z, 0x4140),
                              codes_f16(c.w, 0x4140));
                    st_shared((base + k * 4096) ^ 16, codes_f16(c.x, 0x4342), codes_f16(c.y, 0x4342), codes_f16(c.z, 0x4342),
                              codes_f16(c.w, 0x4342));
                }
            }
            fence_async();
            __syncwarp();
            if (lane == 0) arrive(vals ? v_full(st) : k_full(st));
            at = at_next;
            return true;
        };
        for (int task = cw, i = 0; task < tasks; task += 2 * CONV, i += 2) {
            if (!convert(task, i, raw, coming)) break;
            if (task + CONV >= tasks || !convert(task + CONV, i + 1, coming, raw)) break;
        }
    } else if (n > 0) {  // ------------------------------------------------ MMA issuer
        const uint32_t one = elect_one();
        bool ok = warp_wait(q_full, 0, gone), issued = false;
        const uint64_t q_op = operand(sm + L::q), k_op = operand(sm + L::k), v_op = operand(sm + L::v);
        const auto qk = [&](int q, int j) {
            const uint32_t d = tmem + (2 * q + (j & 1)) * KT;
            const uint64_t qa = q_op + (uint32_t)q * (L::QTILE >> 4), ka = k_op + (uint32_t)(j & (ST - 1)) * (L::TILE >> 4);
            mma_ss<false>(d, qa, ka, idesc(KT), one);
#pragma unroll
            for (int k = 1; k < DH / 16; ++k)
                mma_ss<true>(d, qa + ((k >> 2) * (QT * 128 >> 4) + 2 * (k & 3)), ka + ((k >> 2) * (KT * 128 >> 4) + 2 * (k & 3)),
                             idesc(KT), one);
            issued = true;
            commit(s_full(q, j & 1), one);
        };
        // the logits of two key tiles ahead
        const int nt[2] = {tiles_for(0), tiles_for(1)};
        for (int j = 0; j < 2 && j < n && ok; ++j) {
            if (!(ok = warp_wait(k_full(j), 0, gone))) break;
            fence_after();
            for (int q = 0; q < nq; ++q)
                if (j < nt[q]) qk(q, j);
            commit(k_free(j), one);
        }
        for (int j = 0; j < n && ok; ++j) {
            const int st = j & (ST - 1), ahead = (j + 2) & (ST - 1);
            bool have_v = false, have_k = false;
            for (int q = 0; q < nq; ++q) {
                if (j >= nt[q]) continue;
                if (!(ok = warp_wait(p_full(q, j & 1), (j >> 1) & 1, gone))) break;
                if (!have_v && !(ok = warp_wait(v_full(st), (j / ST) & 1, gone))) break;
                have_v = true;
                fence_after();
                const uint32_t p = tmem + (2 * q + (j & 1)) * KT, o = tmem + L::O + q * DH;
                const uint64_t va = v_op + (uint32_t)st * (L::TILE >> 4);
#pragma unroll
                for (int k = 0; k < KT / 16; ++k) mma_ts(o, p + 8 * k, va + 2 * k, idesc(DH), k > 0 || j > 0, one);
                if (q == nq - 1) commit(v_free(st), one);
                commit(o_done(q), one);
                // a barrier of its own for the last product: the softmax may be up to two
                // phases of o_done away from it, more than a parity tells apart.  Committed
                // last, so that nothing arrives after the tile's rows are out
                if (j == nt[q] - 1) commit(o_last(q), one);
                if (j + 2 < nt[q]) {  // over the buffer that P V read, in order behind it
                    if (!have_k) {
                        if (!(ok = warp_wait(k_full(ahead), ((j + 2) / ST) & 1, gone))) break;
                        have_k = true;
                        fence_after();
                    }
                    qk(q, j + 2);
                    if (q == nq - 1) commit(k_free(ahead), one);
                }
            }
        }
        if (!ok && issued) {  // what was issued ends before the memory is given up
            commit(drain, one);
            bar_wait(drain, 0, KV_WAIT_NS);
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if (warp == MMA_WARP) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
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
        kv_store(a.out, row * a.d + 4 * c, o.x * inv, a.dtype);
        kv_store(a.out, row * a.d + 4 * c + 1, o.y * inv, a.dtype);
        kv_store(a.out, row * a.d + 4 * c + 2, o.z * inv, a.dtype);
        kv_store(a.out, row * a.d + 4 * c + 3, o.w * inv, a.dtype);
    }
    if ((threadIdx.x & 31) == 0 && a.lse) a.lse[row] = l == 0.0f ? -INFINITY : LN2 * (m + log2f(l));
}

template <int DH>
cudaError_t run_prompt(const KvAttnArgs &a, const KvPromptPlan &p, cudaStream_t st) {
    static SmemLimit limit;
    cudaError_t e = limit.launch(kv_prompt_kernel<DH>, Lay<DH>::total, [&] {
        kv_prompt_kernel<DH><<<(unsigned)(p.units * p.splits), Lay<DH>::THREADS, Lay<DH>::total, st>>>(
            a, p.splits, p.splits > 1 ? a.part_cta : nullptr);
    });
    if (e != cudaSuccess || p.splits == 1) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.units * (Lay<DH>::ROWS / 8)));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kv_prompt_join_kernel, a, p.splits, Lay<DH>::ROWS, (const float *)a.part_cta);
    return e != cudaSuccess ? e : launched();
}

}  // namespace

// 16-bit queries and more rows a sequence than a warp tile of k_kv_rows.cu
// holds: at d = 128, 40 rows of 2 sequences that see 900 keys take 22 us here and 24 there, of
// 16 (8 heads) 26 and 46.  d > 128, where this kernel takes longer to start (a CTA
// converts 64 KB of keys and values before its first product is through): not while the
// other one has an SM for every unit and few keys a unit.  At d = 256 (alone in a graph), 40 rows of 16
// sequences, 2 heads (96 units there): 905 keys 26.7 us here and 21.7 there, 1280 24.8 and 25.3, 1400 26.1 and
// 26.3, 1905 28.2 and 32.1; 16 sequences, 8 heads, 905 keys 35 and 62.  Of 12 units the other one stays ahead (1905 keys
// 24.8 and 18.5, in shared stretches), which the rule does not use.
bool kv_prompt_ok(int dtype, int nb, int heads, int d, int64_t rows, int64_t span) {
    if (dtype == SKM_DTYPE_F32 || rows <= KV_ROWS_MOST) return false;
    return d <= 128 || span > 1280 || (int64_t)nb * heads * cdiv(rows, (int64_t)16) > KV_SMS;
}

// Keys a split has at least: a second kernel joins the parts (with 256, 96 rows that
// see 512 keys took 21 us instead of 17; with 512, 40 rows that see 1045 32 instead of 28)
constexpr int64_t SPLIT_KEYS = 320;

size_t kv_prompt_part_most(int d, int64_t span) {
    return span < 2 * SPLIT_KEYS ? 0 : (size_t)KV_SMS * prompt_part(d <= 128 ? Lay<128>::ROWS : Lay<256>::ROWS, d) * 4;
}

KvPromptPlan kv_prompt_plan(int nb, int heads, int group, int d, int max_tokens, int64_t span) {
    KvPromptPlan p = {};
    const int unit_rows = d <= 128 ? Lay<128>::ROWS : Lay<256>::ROWS;
    p.max_tiles = (int)cdiv((int64_t)max_tokens * group, unit_rows);
    p.units = (int64_t)nb * heads * p.max_tiles;
    p.splits = 1;
    // one CTA an SM: split the keys while CTAs are missing
    const int64_t room = KV_SMS / p.units, worth = span / SPLIT_KEYS;
    p.splits = (int)(room < 1 || worth < 1 ? 1 : (room < worth ? room : worth));
    p.part = p.splits > 1 ? (size_t)p.units * p.splits * prompt_part(unit_rows, d) * 4 : 0;
    return p;
}

cudaError_t launch_kv_prompt(const KvAttnArgs &a, const KvPromptPlan &p, cudaStream_t st) {
    return a.d <= 64 ? run_prompt<64>(a, p, st) : a.d <= 128 ? run_prompt<128>(a, p, st) : run_prompt<256>(a, p, st);
}

}  // namespace skm
