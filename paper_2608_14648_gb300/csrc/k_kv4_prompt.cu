// Attention over the 4-bit cache for many query rows (prompt chunks) on tcgen05: 16-bit
// queries.
//
// As k_kv_prompt.cu: a CTA takes 256 query rows of one sequence and key/value head as two tiles of 128
// (d > 128: one), and walks the keys they see in tiles of 64 positions; softmax warps of one
// thread a row, converter warps, a warp for each row tile that issues its products.  Unlike there the
// values' operands hold whole values, so l = sum p, and a tile's sum of weights
// tells whether the reference m has to move.  Operands take one of four forms:
//   ROUNDED  b + s c with one rounding to f16, 2^-11 (bf16 outputs without log-sum-exps, which do not show it): p = 2^(f S - m)
//   SPLIT    (bf16 with log-sum-exps, d <= 128) s (c - 8) as the sum of two f16, a second operand beside the first.  Keys: b + 8 s
//            as b + 4 s + 4 s in 16 dims more, beside the row's sum in two f16: exact.  Values: b + 8 s rounded to f16 and added to
//            the second operand with a rounding.  Twice the products and no more softmax
//   FINE     (f16 outputs, d <= 128) keys as in SPLIT; values s (c - 7.5) in two f16, and b + 7.5 s in fp32, p times it summed in
//            the softmax; weights in two f16, a third product for the second
//   SCALED   (d > 128, where SPLIT has no room) keys: codes less 8, exact, and t = f (s <q, c - 8> + (b + 8 s) sum q) in the
//            softmax, two more operations a logit; values as in ROUNDED, but weights in two f16, a second operand too
// f16 weights and f16 values are each as far off as an f16 output.  Off an exact result, in units of the output's rounding to f16
// (1000 keys; 16000 in one CTA): FINE 1.00 and 1.04, SCALED 1.36 and 1.49, SPLIT for f16 outputs 1.41 and 1.44.  What grows with the
// keys are the sums on tensor cores, which lose half a last bit to every product; codes less 7.5 keep them around 0 (less 8: 2.8 at 16000).
// Prompts of up to 4096, 16 heads of 64: 113 us ROUNDED, 131 SPLIT, 170 FINE, 175 SCALED (with weights in one f16).  4 x 2048 tokens, 32
// query heads on 8 of 128 dims: 176 us ROUNDED, 329 SPLIT (six converter warps and two stages, as shared memory allows, make
// twice the operands), 391 FINE, 288 SCALED, whose values are rounded; 16 on 8 of 192 dims: 263 ROUNDED, 312 SCALED.
//
// What bounds it: the tensor cores, and what keeps them waiting.  A tile of 128 rows and 64 keys of 128 dims takes
// 4 MFLOP; chunks of up to 2048 tokens behind 6144 (two sequences), 32 query heads on 8 of 128 dims, bf16: 270 us, 66% of cuBLAS's bf16 rate.  A
// step's waits were most of what could be gained: one barrier for all that its products need (299 -> 296 us), waits that
// suspend instead of spinning in the schedulers that convert (296 -> 276), constants in registers (276 -> 270).  The
// products alone, issued without a pause, take 74% of that time: one with 64 keys as its columns takes 48 clocks where 32
// would do, and tiles of 128 keys find no room in TMEM beside two row tiles' sums and next logits.
#include "skm_kv_prompt.cuh"

namespace skm {

namespace {

constexpr float TILE_MOST = 65000.0f;  // a tile's sum of weights: above it one may pass the largest f16
// tiles whose absent blocks are noted: a key stage is free once both row tiles' products are through, which are issued
// when their softmax has handed over the tile two before: tile j + ST comes while it reads tile j - 1 at the earliest, 5 behind
constexpr int INFO = 8;

// The forms of operands (above)
enum Keys { ROUNDED, SPLIT, FINE, SCALED };

// DH: dims, padded to 64, 128 or 256
template <int DH, Keys KEYS>
struct Lay {
    static constexpr int NQ = DH <= 128 ? 2 : 1;      // row tiles of a CTA
    static constexpr bool TWO = KEYS == SPLIT || KEYS == FINE;  // keys and values in two operands
    static constexpr bool LOW = KEYS == FINE || KEYS == SCALED;  // weights in two
    static constexpr int ST = DH == 64 || (DH == 128 && !TWO) ? 4 : 2;  // K and V tiles in flight
    static constexpr int ROWS = NQ * QT;
    static_assert(ROWS == prompt_rows(DH));
    // converter warps.  A barrier's parity tells a phase from the next one only, so a warp may not come to a stage two rounds
    // early: from a task to its next one it goes on by no more stages than there are, and for the first one it has
    // waited until its stage was free.  (And no fewer than two stages: a warp's values of tile j would wait for the product
    // of tile j - 1, that one for the keys of tile j + 1, which come after.)
    static constexpr int CONV = NQ == 1 ? 7 : ST == 4 ? 10 : 6;
    static_assert(ST >= 2 && (CONV + KBLK - 1) / KBLK <= ST);
    static constexpr int CONV_WARP0 = 4 * NQ, MMA_WARP = CONV_WARP0 + CONV, THREADS = 32 * (MMA_WARP + NQ);
    // two row tiles: registers of a softmax thread and of the others, no more in all than the 96 or 128 each that the launch comes with
    static constexpr int SOFT_REGS = THREADS == 640 ? 144 : 168, REST_REGS = THREADS == 640 ? 64 : 88;
    // (a quarter of the SM holds a quarter of the warps, rounded up, so a launch of 18 warps comes with the registers of one of 20)
    static constexpr int LAUNCH_REGS = 65536 / ((THREADS + 127) / 128 * 128) / 8 * 8;
    static_assert(NQ == 1 || CONV_WARP0 * SOFT_REGS + (THREADS / 32 - CONV_WARP0) * REST_REGS <= THREADS / 32 * LAUNCH_REGS);
    static constexpr int QTILE = QT * DH * 2, TILE = KT * DH * 2;  // bytes of an operand of rows, of keys or values
    // TWO: rests of keys and values behind them; rows' sums and keys' biases in 16 of 64 dims, those of the two row
    // tiles and of the stages in the same rows
    static constexpr int QMORE = TWO ? QT * 128 : 0, KMORE = TWO ? KT * 128 : 0;
    static constexpr int KTILE = TWO ? 2 * TILE : TILE, VTILE = KTILE;
    static_assert(!TWO || (NQ <= 4 && ST <= 4));
    static constexpr int q = 0, more = NQ * QTILE, kmore = more + QMORE, k = kmore + KMORE, v = k + ST * KTILE, bars = v + ST * VTILE;
    static constexpr int slots = bars + 8 * (6 * ST + 10);  // TMEM address, a flag, the part's index
    static constexpr int wild = (slots + 24 + 15) / 16 * 16;  // a byte a row: its query holds infinities or NaN
    static constexpr int there = wild + ROWS;  // a byte a block of the last INFO tiles: its page is present
    // [INFO][64 keys]: (SCALED) the key's scale and its value at code 8, (FINE) the value at code 7.5
    static constexpr int KEYED = KEYS == SCALED ? 2 * KT : KEYS == FINE ? KT : 0;
    static constexpr int keys = (there + INFO * KBLK + 63) / 64 * 64;
    static constexpr int scales = keys + INFO * KEYED * 4;  // [converter warp][value scales, biases of 16 tokens]
    // one CTA an SM: it takes all of TMEM
    static constexpr int bytes = scales + CONV * 64 + 1024, total = bytes > 120 * 1024 ? bytes : 120 * 1024;
    static_assert(total <= 227 * 1024);
    static constexpr uint32_t O = NQ * 2 * KT;  // TMEM column of O0
};

__device__ __forceinline__ void ld32(uint32_t addr, uint32_t *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void ld_wait32(uint32_t *v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
                   "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                   "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :
                 : "memory");
}

// Bounded, cut short when another role gave up, by a whole warp with one answer.  Suspended meanwhile, a millisecond at a
// time (a loop of short tries took a sixth of the kernel's issue slots)
__device__ __forceinline__ bool warp_sleep(uint32_t b, uint32_t parity, volatile int32_t *gone, const KvAttnArgs &a) {
    const auto there = [&](uint32_t ns) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}\n"
            : "=r"(ok)
            : "r"(b), "r"(parity), "r"(ns)
            : "memory");
        return __all_sync(0xffffffffu, ok);
    };
    if (there(1000000)) return true;
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    while (!there(1000000)) {
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
        if (__any_sync(0xffffffffu, *gone || t - t0 > a.wait_ns)) {
            *gone = 1;
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ __half2 h2(uint32_t x) { return *reinterpret_cast<const __half2 *>(&x); }
__device__ __forceinline__ uint32_t u2(__half2 x) { return *reinterpret_cast<const uint32_t *>(&x); }
// The codes in bits 0..3 and 16..19 of a word, or (HIGH) 4..7 and 20..23, from f16 bits: 1024 + c (1024 + 16 c).  The
// constants in registers: as immediates the two of one logical operation make it two (a third of the
// converters' logical operations)
struct Dequant {
    uint32_t up, down, part, less, mid, mid_part, centre, centre_part;  // f16 pairs: 1024, -1024, 1/16, -64, -1032, -72, -7.5, -71.5
    __device__ __forceinline__ Dequant() {
        asm volatile("mov.b32 %0, 0x64006400;\n\tmov.b32 %1, 0xe400e400;\n\tmov.b32 %2, 0x2c002c00;\n\tmov.b32 %3, 0xd400d400;\n\t"
                     "mov.b32 %4, 0xe408e408;\n\tmov.b32 %5, 0xd480d480;\n\tmov.b32 %6, 0xc780c780;\n\tmov.b32 %7, 0xd478d478;"
                     : "=r"(up), "=r"(down), "=r"(part), "=r"(less), "=r"(mid), "=r"(mid_part), "=r"(centre), "=r"(centre_part));
    }
    template <bool HIGH>
    __device__ __forceinline__ __half2 bits(uint32_t w) const {
        uint32_t x;
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w), "n"(HIGH ? 0x00f000f0 : 0x000f000f), "r"(up));  // and, or
        return h2(x);
    }
    // c - 8, exactly
    template <bool HIGH>
    __device__ __forceinline__ uint32_t codes(uint32_t w) const {
        const __half2 x = bits<HIGH>(w);
        return u2(HIGH ? __hfma2(x, h2(part), h2(mid_part)) : __hadd2(x, h2(mid)));
    }
    // c - 7.5, exactly
    template <bool HIGH>
    __device__ __forceinline__ uint32_t centred(uint32_t w) const {
        const __half2 x = bits<HIGH>(w);
        return u2(HIGH ? __hfma2(x, h2(part), h2(centre_part)) : __hadd2(__hadd2(x, h2(down)), h2(centre)));
    }
    // b + s c with one rounding.  BIG: no more than f16's largest number
    template <bool HIGH, bool BIG>
    __device__ __forceinline__ uint32_t values(uint32_t w, __half2 s, __half2 b) const {
        const __half2 x = bits<HIGH>(w);
        const __half2 c = HIGH ? __hfma2(x, h2(part), h2(less)) : __hadd2(x, h2(down));
        const __half2 v = __hfma2(c, s, b);
        return u2(BIG ? __hmin2(v, h2(0x7bff7bffu)) : v);
    }
};

template <int DH, Keys KEYS>
__global__ void __launch_bounds__(Lay<DH, KEYS>::THREADS, 1)
    kv4_prompt_kernel(const __grid_constant__ KvAttnArgs a, int splits, float *parts) {
    using L = Lay<DH, KEYS>;
    constexpr int ST = L::ST, CONV = L::CONV, ROWS = L::ROWS, CONV_WARP0 = L::CONV_WARP0, MMA_WARP = L::MMA_WARP, THREADS = L::THREADS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // (a warp's number from one lane: the issuing warps' operands then are in uniform registers)
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    uint8_t *smem = smem_raw + ((1024 - (su32(smem_raw) & 1023)) & 1023);  // swizzle atoms
    const uint32_t sm = su32(smem);
    const auto bar = [&](int i) { return sm + L::bars + 8 * i; };
    // Everything that the products of step (row tile q, key tile j) wait for arrives at one barrier: the weights of (q, j),
    // the values of tile j, the keys of tile j + 2.  Logits of (q, j) there: and P V of tile j - 2, in order before them
    const auto k_first = [&](int j) { return bar(j); };  // the keys of the first two tiles
    const auto k_free = [&](int q, int s) { return bar(2 + q * ST + s); };
    const auto v_free = [&](int q, int s) { return bar(2 + 2 * ST + q * ST + s); };
    const auto ready = [&](int q, int s) { return bar(2 + 4 * ST + q * ST + s); };
    const auto s_full = [&](int q, int buf) { return bar(2 + 6 * ST + 2 * q + buf); };
    const auto q_full = [&](int q) { return bar(6 + 6 * ST + q); };
    const auto drain = [&](int q) { return bar(8 + 6 * ST + q); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::slots);
    volatile int32_t *gone = reinterpret_cast<volatile int32_t *>(smem + L::slots + 4);

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
        const auto init = [&](uint32_t b, int count) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(count) : "memory");
        };
        // (one arrival more where a test wants the wait to run out)
        for (int i = 0; i < 2; ++i) init(k_first(i), KBLK + (2 * (int)blockIdx.x + i == a.stuck));
        for (int q = 0; q < L::NQ; ++q) {
            for (int i = 0; i < ST; ++i) init(k_free(q, i), 1), init(v_free(q, i), 1), init(ready(q, i), 4 + 2 * KBLK);
            init(s_full(q, 0), 1), init(s_full(q, 1), 1), init(q_full(q), 4), init(drain(q), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *gone = 0;
    }
    if (a.d < DH) {  // dims from d on are zeros
        for (int i = tid * 16; i < ST * (L::KTILE + L::VTILE); i += THREADS * 16) st_shared(sm + L::k + i, 0, 0, 0, 0);
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
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);

    if constexpr (L::NQ == 2) {
        if (warp < CONV_WARP0) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFT_REGS));
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::REST_REGS));
    }
    if (warp < CONV_WARP0) {  // ------------------------------------------ softmax
        const int q = warp >> 2, row = (warp & 3) * 32 + lane, r = r0 + q * QT + row, nt = tiles_for(q);
        const bool in = r < rows;
        // TWO: rows of at most 2^7, so that their sums are f16's
        float row_sum = 0.0f;
        const float fac = load_rows<DH, KEYS != ROUNDED, L::TWO ? 6 : 15>(a, s, h, r0 + q * QT, (warp & 3) * 32, sm + L::q + q * L::QTILE,
                                                                                 lane, smem + L::wild + q * QT, &row_sum);
        if constexpr (L::TWO) {  // the sum in two f16, three times each, for (b, 4 s, 4 s) of a key twice
            const __half top = __float2half_rn(row_sum), rest = __float2half_rn(row_sum - __half2float(top));
            const uint32_t to = sm + L::more + row * 128;
            st_shared(to + ((2 * q ^ (row & 7)) << 4), u2(__halves2half2(top, top)), u2(__halves2half2(top, rest)), u2(__halves2half2(rest, rest)), 0);
            st_shared(to + (((2 * q + 1) ^ (row & 7)) << 4), 0, 0, 0, 0);
        }
        row_sum *= fac;
        fence_async();
        __syncwarp();
        if (lane == 0) arrive(q_full(q));
        // (rows past the end see everything, with no weight: they slow no one down)
        const int hi = in ? last_of(a, s, r) : 0x7ffffffe, lo = in ? first_of(a, s, r) : 0;
        // rows of the warp see [low, high] whole
        const int high = __shfl_sync(0xffffffffu, hi, 0), low = __reduce_max_sync(0xffffffffu, lo);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t S0 = tmem + lanes + q * 2 * KT, O = tmem + lanes + L::O + q * DH;
        float m = in ? M_NONE : -M_NONE, l = 0.0f;
        [[maybe_unused]] float ob = 0.0f;  // (FINE) the sum of weights times values at code 7.5
        bool ok = true;
        const volatile uint32_t *there = reinterpret_cast<const volatile uint32_t *>(smem + L::there);
        for (int j = 0; j < nt; ++j) {
            const uint32_t S = S0 + (j & 1) * KT;
            if (!(ok = warp_sleep(s_full(q, j & 1), (j >> 1) & 1, gone, a))) break;
            fence_after();
            uint32_t v[KT];
            ld32(S, v);
            ld32(S + 32, v + 32);
            const uint32_t blocks = there[j & (INFO - 1)];
            const int c0 = (t0 + j) * KT;
            const bool whole = c0 >= low && c0 + KT - 1 <= high && blocks == 0x01010101u;
            // the positions of half a tile that the row sees, as bits (opaque, so that it stays in the branches that ask)
            const auto visible = [&](int k0) {
                uint32_t bits = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    int at = c0 + k0 + k * KV_B;
                    asm volatile("" : "+r"(at));
                    const uint32_t sees = ((1u << kv_clamp(hi + 1 - at, 0, KV_B)) - 1) & ~0u << kv_clamp(lo - at, 0, KV_B);
                    if (blocks >> (k0 / 2 + 8 * k) & 1) bits |= sees << (KV_B * k);
                }
                return bits;
            };
            uint32_t P[KT / 2];
            [[maybe_unused]] uint32_t low_bits[L::LOW ? KT / 2 : 1];  // what is left of the weights
            uint64_t sum[4] = {0, 0, 0, 0};
            [[maybe_unused]] float2 mids = make_float2(0.0f, 0.0f);
            // (SCALED) a key's scale and its value at code 8; (FINE) a value's at code 7.5
            const float *scale = reinterpret_cast<const float *>(smem + L::keys) + (j & (INFO - 1)) * L::KEYED;
            // weights of 32 logits
            const auto weigh = [&](auto masked, int k0, uint32_t sees) {
                const float2 f = make_float2(fac, fac), qs = make_float2(row_sum, row_sum), c = make_float2(-m, -m);
                [[maybe_unused]] float4 s4[2], b4[2];  // of four keys, read while the four before are weighed
                if constexpr (L::KEYED > 0) s4[0] = *reinterpret_cast<const float4 *>(scale + k0);
                if constexpr (KEYS == SCALED) b4[0] = *reinterpret_cast<const float4 *>(scale + KT + k0);
#pragma unroll
                for (int i = k0; i < k0 + 32; i += 4) {
                    [[maybe_unused]] const int now = (i >> 2) & 1;
                    if (i + 4 < k0 + 32) {
                        if constexpr (L::KEYED > 0) s4[now ^ 1] = *reinterpret_cast<const float4 *>(scale + i + 4);
                        if constexpr (KEYS == SCALED) b4[now ^ 1] = *reinterpret_cast<const float4 *>(scale + KT + i + 4);
                    }
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        const float2 x = make_float2(__uint_as_float(v[i + k]), __uint_as_float(v[i + k + 1]));
                        float2 t;
                        if constexpr (KEYS == SCALED) {
                            const float2 s2 = k ? make_float2(s4[now].z, s4[now].w) : make_float2(s4[now].x, s4[now].y);
                            const float2 b2 = k ? make_float2(b4[now].z, b4[now].w) : make_float2(b4[now].x, b4[now].y);
                            t = fma2(x, mul2(s2, f), fma2(qs, b2, c));
                        } else {
                            t = fma2(x, f, c);
                        }
                        if constexpr (decltype(masked)::value) {
                            t.x = sees & 1u << (i + k - k0) ? t.x : -INFINITY;
                            t.y = sees & 2u << (i + k - k0) ? t.y : -INFINITY;
                        }
                        if constexpr (L::LOW) {
                            const float2 p = make_float2(ex2(t.x), ex2(t.y));
                            sum[(i + k) / 2 & 3] = add2(sum[(i + k) / 2 & 3], joined(p));
                            // (the upper part cut off, not rounded: a logical operation on the way to what is left)
                            const float2 z = make_float2(__uint_as_float(__float_as_uint(p.x) & 0xffffe000u), __uint_as_float(__float_as_uint(p.y) & 0xffffe000u));
                            P[(i + k) / 2] = pack(z.x, z.y);
                            low_bits[(i + k) / 2] = pack(p.x - z.x, p.y - z.y);
                            if constexpr (KEYS == FINE) mids = fma2(p, k ? make_float2(s4[now].z, s4[now].w) : make_float2(s4[now].x, s4[now].y), mids);
                        } else {
                            P[(i + k) / 2] = weights2(t.x, t.y, sum[(i + k) / 2 & 3]);
                        }
                    }
                }
                if constexpr (L::LOW) {  // at once, while the other half's logits wait in registers
                    st16(S + k0 / 2, P + k0 / 2);
                    st16(S + KT / 2 + k0 / 2, low_bits + k0 / 2);
                }
            };
            const auto weigh_any = [&](int k0) {
                if (whole) weigh(std::false_type{}, k0, 0u);
                else weigh(std::true_type{}, k0, visible(k0));
            };
            const auto total = [&] {
                const float2 t = halves(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
                return t.x + t.y;
            };
            bool moves = j == 0;  // the reference: set by the first tile, seldom moved by a later one
            float add = 0.0f;
            ld_wait32(v);
            if (!moves) {
                weigh_any(0);
                ld_wait32(v + 32);
                weigh_any(32);
                add = total();
                moves = __any_sync(0xffffffffu, add > TILE_MOST);
            } else {
                ld_wait32(v + 32);
            }
            if (moves) {
                // the rows' maxima, with them new references, and the weights (again)
                float top = -INFINITY;
#pragma unroll
                for (int k0 = 0; k0 < KT; k0 += 32) {
                    const uint32_t sees = visible(k0);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (sees & 1u << i) {
                            const float x = __uint_as_float(v[k0 + i]);
                            top = fmaxf(top, KEYS == SCALED ? fmaf(x, scale[k0 + i] * fac, row_sum * scale[KT + k0 + i]) : x * fac);
                        }
                }
                const float to = top > m + 8.0f ? top - M_BELOW : m;
                const float g = ex2(m - to);
                m = to;
                l *= g;
                if constexpr (KEYS == FINE) ob *= g;
                if (j > 0) {
                    if (!(ok = warp_sleep(s_full(q, (j + 1) & 1), ((j + 1) >> 1) & 1, gone, a))) break;  // P V of tile j - 1 is through
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
                if constexpr (L::LOW) st_wait();  // (over the weights that are there)
                sum[0] = sum[1] = sum[2] = sum[3] = 0;
                mids = make_float2(0.0f, 0.0f);
                weigh(std::true_type{}, 0, visible(0));
                weigh(std::true_type{}, 32, visible(32));
                add = total();
            }
            l += add;
            if constexpr (KEYS == FINE) ob += mids.x + mids.y;
            if constexpr (!L::LOW) {
#pragma unroll
                for (int k = 0; k < KT / 2; k += 16) st16(S + k, P + k);
            }
            st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) arrive(ready(q, j % ST));
        }
        if (q < nq) {
            if (ok && nt > 0) {
                ok = warp_sleep(s_full(q, (nt + 1) & 1), ((nt + 1) >> 1) & 1, gone, a);
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
                if constexpr (KEYS == FINE) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + ob);
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
                        w[i] = kv_f16_within(x0, x1);
                    }
                }
                uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.out) + at * a.d + 16 * k);
                dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
            if (in && !part && a.lse) a.lse[at] = l == 0.0f ? -INFINITY : LN2 * (m + log2f(l));
        }
    } else if (warp < MMA_WARP) {  // ------------------------------------- converters
        // tasks: the blocks of all tiles, keys and values; warp w takes w, w + CONV, ...
        const int tasks = n * KBLK, cw = warp - CONV_WARP0, bytes = kv4_bytes(a.d);
        constexpr int NV = DH >= 128 ? DH / 64 : 1;  // 16-byte vectors of a lane: (16-dim chunk lane / 8 + 4 k, g = lane % 8)
        const int g = lane & 7, w0 = lane >> 3;
        uint8_t *mine = smem + L::scales + cw * 64;
        const auto look = [&](int task) {  // 32 of the warp's tasks, one a lane
            int at = -1;
            if (task < tasks) {
                const int blk = t0 * KBLK + task;
                if (blk * KV_B <= last && blk * KV_B + KV_B > first) {
                    const int pg = a.table[(int64_t)b * a.cols + a.by_bpp.div(blk)];
                    if (pg >= 0 && pg < a.pages) at = (pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk);
                }
            }
            return at;
        };
        // codes of a block's keys or values; of an absent one zeros
        const auto load = [&](int at, int from, uint4 (&code)[NV]) {
            const uint4 *p = reinterpret_cast<const uint4 *>(a.k + (int64_t)at * bytes + from) + lane;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                code[k] = make_uint4(0, 0, 0, 0);
                if (at >= 0 && 2 * (lane + 32 * k) < a.d) code[k] = __ldg(p + 32 * k);
            }
        };
        // scale and bias of a token's key (0) or value (1); tokens past the sequence's end were never written: zeros
        const auto scale = [&](int at, int task, int t, int which) {
            if (at < 0 || t >= s.len - (t0 * KBLK + task) * KV_B) return 0u;
            return __ldg(reinterpret_cast<const uint32_t *>(a.k + (int64_t)at * bytes + KV_B * a.d) + 2 * t + which);
        };
        uint4 kc[NV], vc[NV];
        uint32_t ks[2], vs;  // of tokens g and g + 8; of token lane % 16
        const auto load_keys = [&](int at, int task) {
            load(at, 0, kc);
            ks[0] = scale(at, task, g, 0), ks[1] = scale(at, task, g + 8, 0);
        };
        const auto load_values = [&](int at, int task) {
            load(at, 8 * a.d, vc);
            vs = scale(at, task, lane & 15, 1);
        };
        int cur = look(cw + CONV * lane);
        int at = __shfl_sync(0xffffffffu, cur, 0);
        load_keys(at, cw);
        load_values(at, cw);
        const auto beyond = [](uint32_t sb) {  // b + 15 s or 8 s above f16's largest number
            const float2 x = __half22float2(h2(sb));
            return fmaxf(fmaf(15.0f, x.x, x.y), 8.0f * x.x) > 65504.0f;
        };
        const Dequant dq;
        // keys: vector (chunk w, g): tokens g and g + 8, 16 dims each: two 16-byte chunks of an operand row of 64
        // dims.  Values: dims 16 w + g and 16 w + g + 8, 16 tokens each
        const uint32_t k_to = sm + L::k + g * 128 + (((w0 & 3) * 2 ^ g) << 4);
        const uint32_t v_to = sm + L::v + (16 * w0 + g) * 128;
        const auto keys = [&](auto big, uint32_t to) {
            [[maybe_unused]] constexpr bool BIG = decltype(big)::value;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (16 * (w0 + 4 * k) >= a.d) break;
                const uint32_t c[4] = {kc[k].x, kc[k].y, kc[k].z, kc[k].w};
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const __half2 s = __low2half2(h2(ks[t])), b = __high2half2(h2(ks[t]));
                    uint32_t x[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (KEYS == ROUNDED) {
                            x[2 * i] = dq.values<false, BIG>(c[i] >> 8 * t, s, b);
                            x[2 * i + 1] = dq.values<true, BIG>(c[i] >> 8 * t, s, b);
                        } else {
                            x[2 * i] = dq.codes<false>(c[i] >> 8 * t);
                            x[2 * i + 1] = dq.codes<true>(c[i] >> 8 * t);
                        }
                    }
                    if constexpr (L::TWO) {  // s (c - 8) in f16, and what its rounding left (s c at most twice f16's range)
                        uint32_t rest[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            __half2 y = __hmul2(h2(x[i]), s);
                            if constexpr (BIG) y = __hmax2(__hmin2(y, h2(0x7bff7bffu)), h2(0xfbfffbffu));
                            rest[i] = u2(__hfma2(h2(x[i]), s, __hneg2(y)));
                            x[i] = u2(y);
                        }
                        st_shared(to + L::TILE + k * (KT * 128) + t * 1024, rest[0], rest[1], rest[2], rest[3]);
                        st_shared((to + L::TILE + k * (KT * 128) + t * 1024) ^ 16, rest[4], rest[5], rest[6], rest[7]);
                    }
                    st_shared(to + k * (KT * 128) + t * 1024, x[0], x[1], x[2], x[3]);
                    st_shared((to + k * (KT * 128) + t * 1024) ^ 16, x[4], x[5], x[6], x[7]);
                }
            }
        };
        const auto values = [&](auto big, uint32_t to) {
            constexpr bool BIG = decltype(big)::value;
#pragma unroll
            for (int half = 0; half < 2; ++half) {  // tokens 0 .. 7, 8 .. 15
                const uint4 s4 = *reinterpret_cast<const uint4 *>(mine + 16 * half), b4 = *reinterpret_cast<const uint4 *>(mine + 32 + 16 * half);
                const uint32_t s[4] = {s4.x, s4.y, s4.z, s4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (16 * (w0 + 4 * k) >= a.d) break;
                    const uint32_t c[4] = {vc[k].x, vc[k].y, vc[k].z, vc[k].w};
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        uint32_t x[4];
                        if constexpr (L::TWO) {  // s (c - 8) in f16; what is left, exactly, and the value at code 8 in one.  FINE: s (c - 7.5),
                                                // exactly but for 2^-25 where s is below 2^-13
                            uint32_t rest[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t w = c[i] >> 8 * t;
                                const __half2 u = h2(KEYS == FINE ? (half ? dq.centred<true>(w) : dq.centred<false>(w)) : half ? dq.codes<true>(w) : dq.codes<false>(w));
                                __half2 y = __hmul2(u, h2(s[i]));
                                if constexpr (BIG) y = __hmax2(__hmin2(y, h2(0x7bff7bffu)), h2(0xfbfffbffu));
                                const __half2 left = __hfma2(u, h2(s[i]), __hneg2(y));
                                rest[i] = u2(KEYS == SPLIT ? __hadd2(left, h2(b[i])) : left);
                                x[i] = u2(y);
                            }
                            st_shared((to + L::TILE + k * 8192 + t * 1024) ^ (16 * half), rest[0], rest[1], rest[2], rest[3]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                x[i] = half ? dq.values<true, BIG>(c[i] >> 8 * t, h2(s[i]), h2(b[i])) : dq.values<false, BIG>(c[i] >> 8 * t, h2(s[i]), h2(b[i]));
                        }
                        st_shared((to + k * 8192 + t * 1024) ^ (16 * half), x[0], x[1], x[2], x[3]);
                    }
                }
            }
        };
        // A stage is free when the row tiles that go through its tile are through with it: even lanes ask the first one's
        // barrier, odd ones the second's
        const int ask = nq == 2 ? lane & 1 : 0, nt0 = tiles_for(0);
        for (int task = cw, i = 0; task < tasks; task += CONV, ++i) {
            const int j = task / KBLK, st = j % ST, blk = task & (KBLK - 1);
            if ((i & 31) == 31) cur = look(task + CONV * (1 + lane));
            const int at_next = __shfl_sync(0xffffffffu, cur, (i + 1) & 31);
            const bool big = __any_sync(0xffffffffu, beyond(vs) || (KEYS != SCALED && (beyond(ks[0]) || beyond(ks[1]))));
            const int whose = j - ST < nt0 ? ask : nq - 1;
            if (!warp_sleep(k_free(whose, st), ((j / ST) & 1) ^ 1, gone, a)) break;
            if (lane == 0) smem[L::there + (j & (INFO - 1)) * KBLK + blk] = at >= 0;
            if (L::TWO && lane < KV_B) {  // (b, 4 s, 4 s) twice: eight s, but in f16's range
                const __half2 sb = h2(ks[lane >> 3]);
                const __half b = __high2half(sb), s4 = __hmul(__low2half(sb), __ushort_as_half(0x4400));
                const uint32_t to = sm + L::kmore + (blk * KV_B + lane) * 128;
                st_shared(to + ((2 * st ^ (lane & 7)) << 4), u2(__halves2half2(b, s4)), u2(__halves2half2(s4, b)), u2(__halves2half2(s4, s4)), 0);
                st_shared(to + (((2 * st + 1) ^ (lane & 7)) << 4), 0, 0, 0, 0);
            }
            if (KEYS == FINE && lane < KV_B) {
                const float2 sb = __half22float2(h2(vs));
                reinterpret_cast<float *>(smem + L::keys)[(j & (INFO - 1)) * L::KEYED + blk * KV_B + lane] = fmaf(7.5f, sb.x, sb.y);
            }
            if (KEYS == SCALED && lane < 8) {
                float *scale = reinterpret_cast<float *>(smem + L::keys) + (j & (INFO - 1)) * 2 * KT + blk * KV_B + g;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float2 sb = __half22float2(h2(ks[t]));
                    scale[8 * t] = sb.x;
                    scale[KT + 8 * t] = fmaf(8.0f, sb.x, sb.y);
                }
            }
            if (KEYS != SCALED && big) keys(std::true_type{}, k_to + st * L::KTILE + blk * 2048);
            else keys(std::false_type{}, k_to + st * L::KTILE + blk * 2048);
            fence_async();
            __syncwarp();
            if (j < 2) {
                if (lane == 0) arrive(k_first(j));
            } else if (lane < L::NQ) {
                arrive(ready(lane, (j - 2) % ST));
            }
            load_keys(at_next, task + CONV);
            if (lane < KV_B) {
                __half bias = __high2half(h2(vs));
                if constexpr (KEYS == SPLIT) bias = __hmin(__hfma(__low2half(h2(vs)), __ushort_as_half(0x4800), bias), __ushort_as_half(0x7bff));  // + 8 s
                reinterpret_cast<uint16_t *>(mine)[lane] = (uint16_t)vs;
                reinterpret_cast<__half *>(mine)[KV_B + lane] = bias;
            }
            __syncwarp();
            if (!warp_sleep(v_free(whose, st), ((j / ST) & 1) ^ 1, gone, a)) break;
            if (big) values(std::true_type{}, v_to + st * L::VTILE + ((blk * 2 ^ g) << 4));
            else values(std::false_type{}, v_to + st * L::VTILE + ((blk * 2 ^ g) << 4));
            fence_async();
            __syncwarp();
            // (the last two tiles' steps wait for no keys: once more in their place)
            if (lane < L::NQ) {
                arrive(ready(lane, st));
                if (j + 2 >= n) arrive(ready(lane, st));
            }
            load_values(at_next, task + CONV);
            at = at_next;
        }
    } else {  // -------------------------------------------------------- MMA issuer of a row tile
        // (one a row tile: between its products a warp waits, commits and counts for as long as the products take)
        const int q = warp - MMA_WARP, nt = tiles_for(q);
        const uint32_t one = elect_one();
        bool ok = nt > 0 && warp_sleep(q_full(q), 0, gone, a), issued = false;
        const uint64_t q_op = operand(sm + L::q + q * L::QTILE), k_op = operand(sm + L::k), v_op = operand(sm + L::v);
        const uint32_t S = tmem + 2 * q * KT, O = tmem + L::O + q * DH;
        const auto qk = [&](int j) {
            const uint32_t d = S + (j & 1) * KT;
            const uint64_t ka = k_op + (uint32_t)(j % ST) * (L::KTILE >> 4);
            const auto dims = [&](auto add, uint64_t kb) {
                mma_ss<decltype(add)::value>(d, q_op, kb, idesc(KT), one);
#pragma unroll
                for (int k = 1; k < DH / 16; ++k)
                    mma_ss<true>(d, q_op + ((k >> 2) * (QT * 128 >> 4) + 2 * (k & 3)), kb + ((k >> 2) * (KT * 128 >> 4) + 2 * (k & 3)),
                                 idesc(KT), one);
            };
            dims(std::false_type{}, ka);
            if constexpr (L::TWO) {
                dims(std::true_type{}, ka + (L::TILE >> 4));
                mma_ss<true>(d, operand(sm + L::more) + 2 * q, operand(sm + L::kmore) + 2 * (j % ST), idesc(KT), one);
            }
            issued = true;
            commit(k_free(q, j % ST), one);
        };
        // the logits of two key tiles ahead
        for (int j = 0; j < 2 && j < nt && ok; ++j) {
            if (!(ok = warp_sleep(k_first(j), 0, gone, a))) break;
            fence_after();
            qk(j);
            commit(s_full(q, j), one);
        }
#pragma unroll 1
        for (int j = 0; j < nt && ok; ++j) {
            if (!(ok = warp_sleep(ready(q, j % ST), (j / ST) & 1, gone, a))) break;
            fence_after();
            const uint32_t p = S + (j & 1) * KT;
            const uint64_t va = v_op + (uint32_t)(j % ST) * (L::VTILE >> 4);
#pragma unroll
            for (int k = 0; k < KT / 16; ++k) mma_ts(O, p + 8 * k, va + 2 * k, idesc(DH), k > 0 || j > 0, one);
            const auto more = [&](uint32_t w, uint64_t v) {
#pragma unroll
                for (int k = 0; k < KT / 16; ++k) mma_ts(O, p + w + 8 * k, v + 2 * k, idesc(DH), 1, one);
            };
            if constexpr (L::TWO) more(0, va + (L::TILE >> 4));  // the values' rests
            if constexpr (L::LOW) more(KT / 2, va);  // the weights'
            commit(v_free(q, j % ST), one);
            if (j + 2 < nt) qk(j + 2);  // over the buffer that P V read, in order behind it
            commit(s_full(q, j & 1), one);
        }
        if (nt > 0 && !ok && issued) {  // what was issued ends before the memory is given up
            commit(drain(q), one);
            bar_wait(drain(q), 0, KV_WAIT_NS);
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

template <int DH, Keys KEYS>
cudaError_t run_prompt(const KvAttnArgs &a, const KvPromptPlan &p, cudaStream_t st) {
    static SmemLimit limit;
    cudaError_t e = limit.launch(kv4_prompt_kernel<DH, KEYS>, Lay<DH, KEYS>::total, [&] {
        kv4_prompt_kernel<DH, KEYS><<<(unsigned)(p.units * p.splits), Lay<DH, KEYS>::THREADS, Lay<DH, KEYS>::total, st>>>(
            a, p.splits, p.splits > 1 ? a.part_cta : nullptr);
    });
    if (e != cudaSuccess || p.splits == 1) return e;
    return run_prompt_join(a, p, Lay<DH, KEYS>::ROWS, st);
}

}  // namespace

cudaError_t launch_kv4_prompt(const KvAttnArgs &a, const KvPromptPlan &p, cudaStream_t st) {
    // bf16 outputs hide the rounding of keys (both 1.7e-3 off); f16 ones and log-sum-exps would show it
    if (a.dtype == SKM_DTYPE_BF16 && !a.lse)
        return a.d <= 64 ? run_prompt<64, ROUNDED>(a, p, st) : a.d <= 128 ? run_prompt<128, ROUNDED>(a, p, st) : run_prompt<256, ROUNDED>(a, p, st);
    if (a.d > 128) return run_prompt<256, SCALED>(a, p, st);
    if (a.dtype == SKM_DTYPE_BF16) return a.d <= 64 ? run_prompt<64, SPLIT>(a, p, st) : run_prompt<128, SPLIT>(a, p, st);
    return a.d <= 64 ? run_prompt<64, FINE>(a, p, st) : run_prompt<128, FINE>(a, p, st);
}

}  // namespace skm
