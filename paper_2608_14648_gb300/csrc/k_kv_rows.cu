// Attention over the 8-bit cache for few query rows (single tokens, a few
// tokens): one row tile a head, whose codes cross HBM once, and everything else hides behind
// them.  (More rows than a tile, fp32 ones or 16-bit ones of d > 128: each tile fetches them again.)
//
// Work.  A unit is a sequence's tile of RT query rows (token-major, then the
// heads of one group) and a key/value head; its blocks of 16 tokens are its
// items.  All items of a launch form one line, units in order (sequence, row
// tile, head), and each CTA takes an equal stretch of it, each warp an equal
// stretch of its CTA's: short and long sequences balance without a plan on the
// host, and a warp crosses at most two cuts.  (With `whole`, a CTA's stretch
// is one unit: few short ones then need no second kernel.)  A warp runs alone: lane 0
// keeps a ring of cp.async.bulk copies (a block's keys and values, 16 d bytes
// each, contiguous in the cache) going across unit boundaries; the table
// entries and scales of 32 items are fetched at once, a window ahead.
//
// Mathematics.  With S = scale log2(e) q.k, codes c and scales s_k, s_v, the
// block's logits are t = S + log2 s_v, S = (scale log2(e) s_k) q.c_k; p = 2^(t - m),
// o = sum p c_v, l = sum p / s_v: the value scale costs one addition a logit
// and o needs none.  m is a running reference that moves only when a logit
// exceeds it by 15 (then to 7 below the maximum), so p < 2^15 and the sums are rarely
// rescaled.  out = o / l, lse = ln2 (m + log2 l).
//
// What bounds it.  Sequences with much to read: HBM (GB300, 8 heads of 128: 64
// sequences of up to 8192 tokens, 485 MB, 99 us = 4.9 TB/s; one of 131079, 269
// MB, 56 us = 4.8 TB/s; a plain copy of as much 6.8).  While all
// warps of the batch run it is read at 6.9 TB/s; they end 62 to 82 us after the start
// (SMs do not all get the same share), some 4 us pass until the first block has arrived
// (lengths, table, scales, each behind the one before), and merging takes the rest.  Short
// sequences: instructions that are fetched for the first time (7 of the 9 us for one of
// 333 tokens, in a graph).
//
// Joining.  Partial (m, l, o) of units that warps share are merged by their
// CTA, those that CTAs share by kv_join_kernel; both in the line's order, so
// the result does not depend on timing.  A CTA that goes on with a unit notes what there is to
// join, so the second kernel has a CTA a cut and row, whatever the batch (with one a unit
// and row, each finding its place, 900 sequences of up to 2501 tokens took 344 us
// instead of 259).
#include <algorithm>
#include <initializer_list>

#include "skm_kv_dev.cuh"

namespace skm {

namespace {

// The line of items.  cum[i] (shared memory): items of sequences before b0 + i.
struct Line {
    const int64_t *cum;
    const Seq *seq;
    int b0, nb;
    __device__ __forceinline__ int find(int64_t item) const {  // the sequence that holds an item
        int lo = 0, hi = nb;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cum[mid] <= item) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// CTAs that share W items: no more than leave every warp two items
__host__ __device__ __forceinline__ int64_t active_ctas(int64_t W, int nw, int64_t grid) {
    const int64_t c = (W + 2 * nw - 1) / (2 * nw);
    return c < 1 ? 1 : (c > grid ? grid : c);
}

// 32 items, one a lane.  Three steps, so that the two dependent loads behind
// an item (its page, then the block's scales) are waited for long after they
// were issued: where the item is, its block, its scales to shared memory.
struct Window {
    int pg, at;  // page; block of the pool, -1: nothing to do
    int blk, seq, unit;
    float2 sc;
    uint32_t todo, starts;  // (all lanes the same) items with work, items that begin a unit
    int n;
};

template <int RT>
__device__ __forceinline__ void window_pages(const KvAttnArgs &a, const Line &ln, int64_t base, int64_t end, int lane,
                                             Window &w) {
    w.n = end - base > 32 ? 32 : (int)(end > base ? end - base : 0);
    w.pg = -1;
    w.blk = w.seq = w.unit = 0;
    bool starts = false;
    if (lane < w.n) {
        const int64_t item = base + lane;
        const int b = ln.find(item);
        const Seq s = ln.seq[b];
        const uint64_t rem = (uint64_t)(item - ln.cum[b]);
        uint32_t u, k;
        if (rem >> 32) {
            u = (uint32_t)(rem / (uint32_t)s.cnt);
            k = (uint32_t)(rem % (uint32_t)s.cnt);
        } else {
            u = (uint32_t)rem / (uint32_t)s.cnt;
            k = (uint32_t)rem - u * (uint32_t)s.cnt;
        }
        starts = k == 0;
        w.seq = b;
        w.unit = (int)u;
        w.blk = s.lo + (int)k;
        const int r0 = a.by_heads.div((int)u) * RT, r1 = min(r0 + RT, s.n * a.group) - 1;
        if (w.blk * KV_B <= last_of(a, s, r1) && w.blk * KV_B + KV_B > first_of(a, s, r0))
            w.pg = a.table[(int64_t)(ln.b0 + b) * a.cols + a.by_bpp.div(w.blk)];
    }
    w.starts = __ballot_sync(0xffffffffu, starts);
    w.todo = 0;
}
__device__ __forceinline__ void window_blocks(const KvAttnArgs &a, Window &w) {
    const bool there = w.pg >= 0 && w.pg < a.pages;
    w.at = there ? (w.pg * a.heads + a.by_heads.mod(w.unit)) * a.bpp + a.by_bpp.mod(w.blk) : -1;
    w.sc = there ? a.scales[w.at] : make_float2(0.0f, 0.0f);
    w.todo = __ballot_sync(0xffffffffu, there);
}
__device__ __forceinline__ void window_scales(const Window &w, float4 *mem, int lane) {
    mem[lane] = value_scale(w.sc);
    __syncwarp();
}

// dims 4 c .. 4 c + 3 of an output row
__device__ __forceinline__ void store_row4(const KvAttnArgs &a, int64_t row, int c, float4 o, float inv) {
    o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (a.dtype == SKM_DTYPE_F32) {
        reinterpret_cast<float4 *>(static_cast<float *>(a.out) + row * a.d)[c] = o;
    } else if (a.dtype == SKM_DTYPE_BF16) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(o.x, o.y), y = __floats2bfloat162_rn(o.z, o.w);
        reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row * a.d)[c] =
            make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
    } else {
        const __half2 x = __floats2half2_rn(o.x, o.y), y = __floats2half2_rn(o.z, o.w);
        reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row * a.d)[c] =
            make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
    }
}

// A partial result: RT x (m, l), padded to 16 bytes, then RT rows of d sums.
template <int RT>
__host__ __device__ constexpr int part_head() {
    return (2 * RT + 3) & ~3;
}
template <int RT>
__host__ __device__ __forceinline__ constexpr int64_t part_floats(int d) {
    return part_head<RT>() + (int64_t)RT * d;
}

// Merges parts of one unit: the lanes in `same` hold one each, in order.  A
// warp takes a row: a lane its part's (m, l), then all lanes the row's dims.  To
// the outputs (dst NULL) or as a part again.
template <int RT, int Q>
__device__ __forceinline__ void merge_parts(const KvAttnArgs &a, const float *part, uint32_t same, const Seq &s, int unit,
                                            float *dst, int warp, int warps, int lane) {
    const int d4 = a.d / 4, h = a.by_heads.mod(unit), r0 = a.by_heads.div(unit) * RT;
    const int rows = min(RT, s.n * a.group - r0);
    const bool mine = (same >> lane) & 1;
#pragma unroll 1
    for (int r = warp; r < rows; r += warps) {
        const float2 ml = mine ? *reinterpret_cast<const float2 *>(part + 2 * r) : make_float2(M_NONE, 0.0f);
        float m = ml.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float f = mine ? ex2(ml.x - m) : 0.0f;
        float l = ml.y * f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        float4 o[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) o[q] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (uint32_t bits = same; bits;) {
            float w[4];
            const float4 *p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {  // past the last: the first again, weight 0
                const int j = __ffs(bits ? bits : same) - 1;
                const float fj = __shfl_sync(0xffffffffu, f, j);
                w[k] = bits ? fj : 0.0f;
                p[k] = reinterpret_cast<const float4 *>(
                    __shfl_sync(0xffffffffu, (unsigned long long)part, j) + 4ull * (part_head<RT>() + r * a.d));
                bits &= bits - 1;
            }
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                if (lane + 32 * q >= d4) break;
                float4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = p[k][lane + 32 * q];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    o[q].x = fmaf(v[k].x, w[k], o[q].x), o[q].y = fmaf(v[k].y, w[k], o[q].y);
                    o[q].z = fmaf(v[k].z, w[k], o[q].z), o[q].w = fmaf(v[k].w, w[k], o[q].w);
                }
            }
        }
        const int64_t row = row_index(a, s, h, r0 + r);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (lane + 32 * q >= d4) break;
            if (dst) reinterpret_cast<float4 *>(dst + part_head<RT>() + r * a.d)[lane + 32 * q] = o[q];
            else store_row4(a, row, lane + 32 * q, o[q], inv);
        }
        if (lane == 0) {
            if (dst) dst[2 * r] = m, dst[2 * r + 1] = l;
            else if (a.lse) a.lse[row] = l == 0.0f ? -INFINITY : LN2 * (m + log2f(l));
        }
    }
}

// The positions that a tile's rows see, kept by the warp for its masked blocks
template <int RT>
constexpr int LIMITS = (8 * RT + 15) & ~15;
template <int RT>
__device__ __forceinline__ void limits(const KvAttnArgs &a, const Seq &s, int r0, int2 *lim, int lane) {
    if (lane < RT) lim[lane] = make_int2(last_of(a, s, r0 + lane), first_of(a, s, r0 + lane));
}

// Rows of one warp in fp32 on CUDA cores.  Scores: lane = (half, token), a
// half takes every other 16-dim chunk of the keys; sums: lane = dims lane,
// lane + 32, ...  q and p pass through the warp's shared memory.
template <int R, int DPL>
struct Fp32Rows {
    static constexpr int RT = R, D4 = DPL > 4 ? 2 : 1;
    static constexpr bool ONE_D = false;
    static constexpr size_t __host__ __device__ scratch(int d) { return (size_t)R * (d + KV_B) * 4 + LIMITS<R>; }
    float o[R][DPL], m[R], l[R];
    float *q, *p;
    int2 *lim;

    __device__ __forceinline__ void begin(const KvAttnArgs &a, const Seq &s, int h, int r0, uint8_t *mem,
                                          int lane) {
        lim = reinterpret_cast<int2 *>(mem);
        q = reinterpret_cast<float *>(mem + LIMITS<R>);
        p = q + R * a.d;
        __syncwarp();
        limits<R>(a, s, r0, lim, lane);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = M_NONE, l[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < DPL; ++i) o[r][i] = 0.0f;
            const int rr = r0 + r;
            const bool in = rr < s.n * a.group;
            const int64_t at = in ? (int64_t)(s.row0 + a.by_group.div(rr)) * a.q_token + (int64_t)(h * a.group + a.by_group.mod(rr)) * a.q_head : 0;
            for (int i = lane; i < a.d; i += 32) q[r * a.d + i] = in ? kv_load(a.Q, at + i, a.dtype) * a.scale_log2 : 0.0f;
        }
        __syncwarp();
    }

    __device__ __forceinline__ void block(const KvAttnArgs &a, const uint8_t *K, const uint8_t *V, int blk, float ks, float lvs, float ivs, bool mask, int lane) {
        const int t = lane & 15, half = lane >> 4, nc = a.d / KV_B;
        float x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = 0.0f;
        for (int w = half; w < nc; w += 2) {
            const uint4 c = *reinterpret_cast<const uint4 *>(K + w * 256 + t * 16);
            const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float k0 = kv_code(word[i], 0), k1 = kv_code(word[i], 1), k2 = kv_code(word[i], 2), k3 = kv_code(word[i], 3);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float4 qq = *reinterpret_cast<const float4 *>(q + r * a.d + 16 * w + 4 * i);
                    x[r] = fmaf(k0, qq.x, x[r]);
                    x[r] = fmaf(k1, qq.y, x[r]);
                    x[r] = fmaf(k2, qq.z, x[r]);
                    x[r] = fmaf(k3, qq.w, x[r]);
                }
            }
        }
        const int place = 4 * ((t & 7) >> 1) + 2 * (t >> 3) + (t & 1);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            x[r] += __shfl_xor_sync(0xffffffffu, x[r], 16);
            x[r] = fmaf(x[r], ks, lvs);
            if (mask) {
                const int j = blk * KV_B + t;
                if (j > lim[r].x || j < lim[r].y) x[r] = -INFINITY;
            }
            if (__any_sync(0xffffffffu, x[r] > m[r] + M_SLACK)) {
                float top = x[r];
#pragma unroll
                for (int b = 8; b > 0; b >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
                const float to = top - M_BELOW, f = exp2f(m[r] - to);
                m[r] = to;
                l[r] *= f;
#pragma unroll
                for (int i = 0; i < DPL; ++i) o[r][i] *= f;
            }
            const float e = exp2f(x[r] - m[r]);
            if (half == 0) {
                l[r] = fmaf(e, ivs, l[r]);
                p[r * KV_B + place] = e;
            }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            const int dim = lane + 32 * i;
            if (dim >= a.d) break;
            const uint4 c = *reinterpret_cast<const uint4 *>(V + dim * 16);
            const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float k0 = kv_code(word[w], 0), k1 = kv_code(word[w], 1), k2 = kv_code(word[w], 2), k3 = kv_code(word[w], 3);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float4 pp = *reinterpret_cast<const float4 *>(p + r * KV_B + 4 * w);
                    o[r][i] = fmaf(k0, pp.x, o[r][i]);
                    o[r][i] = fmaf(k1, pp.y, o[r][i]);
                    o[r][i] = fmaf(k2, pp.z, o[r][i]);
                    o[r][i] = fmaf(k3, pp.w, o[r][i]);
                }
            }
        }
        __syncwarp();
    }

    __device__ __forceinline__ void close(int) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int b = 16; b > 0; b >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], b);
    }
    __device__ __forceinline__ void put(const KvAttnArgs &a, float *dst, int lane) const {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (lane == 0) dst[2 * r] = m[r], dst[2 * r + 1] = l[r];
#pragma unroll
            for (int i = 0; i < DPL; ++i)
                if (lane + 32 * i < a.d) dst[part_head<R>() + r * a.d + lane + 32 * i] = o[r][i];
        }
    }
    __device__ __forceinline__ void finish(const KvAttnArgs &a, const Seq &s, int h, int r0, int lane) const {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r0 + r >= s.n * a.group) break;
            const int64_t row = row_index(a, s, h, r0 + r);
            const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
#pragma unroll
            for (int i = 0; i < DPL; ++i)
                if (lane + 32 * i < a.d) kv_store(a.out, row * a.d + lane + 32 * i, o[r][i] * inv, a.dtype);
            if (lane == 0 && a.lse) a.lse[row] = l[r] == 0.0f ? -INFINITY : LN2 * (m[r] + log2f(l[r]));
        }
    }
};

// ---- 16-bit queries: mma.m16n8k16, f16 operands, fp32 sums
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// operand A of a 16 x 16 tile of codes: x rows 0..7, y rows 8..15, four
// consecutive bytes a lane (columns 2c, 2c + 1, 2c + 8, 2c + 9 of the tile)
__device__ __forceinline__ void codes_a(uint32_t x, uint32_t y, uint32_t (&a)[4]) {
    a[0] = codes_f16(x, 0x4140);
    a[1] = codes_f16(y, 0x4140);
    a[2] = codes_f16(x, 0x4342);
    a[3] = codes_f16(y, 0x4342);
}

// 4 values without the alignment of a vector (not inlined: a rare path)
__device__ __noinline__ uint2 load4(const uint16_t *x) {
    return make_uint2(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16);
}
// two bf16 times a power of two as f16
__device__ __forceinline__ uint32_t bf16_f16(uint32_t w, float mul) {
    const __half2 x = __floats2half2_rn(__uint_as_float(w << 16) * mul, __uint_as_float(w & 0xffff0000u) * mul);
    return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ uint16_t bits16(float v, bool bf) {
    return bf ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}

// Rows of one warp on tensor cores, transposed: S^T = K q^T and o^T = V^T p^T
// (16 tokens or dims x 8 rows x 16), so a tile of 8 rows wastes nothing when
// the heads of a group are 8.  Both cache layouts are read by ldmatrix, 512
// consecutive bytes at a time, and a lane's word is the operand's columns: of
// the dims of a 16-dim chunk, lane column c holds 4c .. 4c + 3 (the queries
// are laid out to match); of the tokens, the cache's byte order makes it 2c,
// 2c + 1, 2c + 8, 2c + 9, the operand's own.  p^T comes from S^T by movmatrix.
// bf16 queries become f16 after scaling a row by a power of two (to_f16).
// DC: 16-dim chunks at most (FULL: exactly), NT: tiles of 8 rows.
template <int DC, int NT, bool FULL>
struct MmaRows {
    static constexpr int RT = 8 * NT;
    static constexpr int D4 = DC > 8 ? 2 : 1;
    static constexpr bool ONE_D = FULL;
    static constexpr bool QMEM = NT * DC >= 32;  // the queries' operands wait in shared memory
    static constexpr size_t __host__ __device__ scratch(int) { return (QMEM ? (size_t)NT * DC * 2 * 32 * 4 : 0) + LIMITS<RT>; }
    float o[NT][DC][4], m[NT][2], l[NT][2], fac[NT][2];
    uint32_t q[QMEM ? 1 : NT][QMEM ? 1 : DC][2];
    uint2 *qmem;
    int2 *lim;

    __device__ __forceinline__ void begin(const KvAttnArgs &a, const Seq &s, int h, int r0, uint8_t *mem,
                                          int lane) {
        const int g = lane >> 2, c = lane & 3, nc = FULL ? DC : a.d / KV_B;
        lim = reinterpret_cast<int2 *>(mem);
        qmem = reinterpret_cast<uint2 *>(mem + LIMITS<RT>);
        __syncwarp();
        limits<RT>(a, s, r0, lim, lane);
        const bool bf = a.dtype == SKM_DTYPE_BF16;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int rr = r0 + 8 * t + g;
            const bool in = rr < s.n * a.group;
            const uint16_t *x = static_cast<const uint16_t *>(a.Q);
            if (in) x += (int64_t)(s.row0 + a.by_group.div(rr)) * a.q_token + (int64_t)(h * a.group + a.by_group.mod(rr)) * a.q_head + 4 * c;
            uint2 raw[DC];
#pragma unroll
            for (int w = 0; w < DC; ++w) raw[w] = make_uint2(0, 0);
            if (in && a.q_wide) {
#pragma unroll
                for (int w = 0; w < DC; ++w)
                    if (w < nc) raw[w] = *reinterpret_cast<const uint2 *>(x + 16 * w);
            } else if (in) {
#pragma unroll
                for (int w = 0; w < DC; ++w)
                    if (w < nc) raw[w] = load4(x + 16 * w);
            }
            float mul = 1.0f, back = 1.0f;
            if (bf) {
                uint32_t top = 0;  // the largest |x| as bits (of one sign, they order like the numbers)
#pragma unroll
                for (int w = 0; w < DC; ++w) {
                    top = max(max(top, raw[w].x << 16 & 0x7fff0000u), raw[w].x & 0x7fff0000u);
                    top = max(max(top, raw[w].y << 16 & 0x7fff0000u), raw[w].y & 0x7fff0000u);
                }
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const Pow2 by = to_f16(top >> 23);
                mul = by.mul, back = by.back;
            }
#pragma unroll
            for (int w = 0; w < DC; ++w) {
                const uint32_t b0 = bf ? bf16_f16(raw[w].x, mul) : raw[w].x, b1 = bf ? bf16_f16(raw[w].y, mul) : raw[w].y;
                if constexpr (QMEM) qmem[(t * DC + w) * 32 + lane] = make_uint2(b0, b1);
                else q[t][w][0] = b0, q[t][w][1] = b1;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[t][w][i] = 0.0f;
            }
            back *= a.scale_log2;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fac[t][i] = __shfl_sync(0xffffffffu, back, (2 * c + i) * 4);
                m[t][i] = M_NONE;
                l[t][i] = 0.0f;
            }
        }
        __syncwarp();
    }

    __device__ __forceinline__ void block(const KvAttnArgs &a, const uint8_t *K, const uint8_t *V, int blk, float ks, float lvs, float ivs, bool mask, int lane) {
        const int g = lane >> 2, c = lane & 3, nc = FULL ? DC : a.d / KV_B;
        float x[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = 0.0f;
        const uint32_t ka = su32(K) + lane * 16, va = su32(V) + lane * 16;
#pragma unroll
        for (int w = 0; w < DC; w += 2) {
            if (w >= nc) break;
            uint32_t r[4], f[4];
            ldsm4(ka + w * 256, r);
            codes_a(r[0], r[1], f);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (QMEM) {
                    const uint2 b = qmem[(t * DC + w) * 32 + lane];
                    mma16816(x[t], f, b.x, b.y);
                } else {
                    mma16816(x[t], f, q[t][w][0], q[t][w][1]);
                }
            }
            if (w + 1 >= nc) break;
            codes_a(r[2], r[3], f);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (QMEM) {
                    const uint2 b = qmem[(t * DC + w + 1) * 32 + lane];
                    mma16816(x[t], f, b.x, b.y);
                } else {
                    mma16816(x[t], f, q[t][w + 1][0], q[t][w + 1][1]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float f[2] = {fac[t][0] * ks, fac[t][1] * ks};
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = fmaf(x[t][i], f[i & 1], lvs);
        }
        if (mask) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = blk * KV_B + g + 8 * (i >> 1);
                    const int2 see = lim[8 * t + 2 * c + (i & 1)];
                    if (j > see.x || j < see.y) x[t][i] = -INFINITY;
                }
        }
        float p[NT][4];
        const auto weigh = [&] {  // weights, and the largest sum of two
            float most = 0.0f;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) p[t][i] = ex2(x[t][i] - m[t][i & 1]);
                most = fmaxf(most, fmaxf(p[t][0] + p[t][2], p[t][1] + p[t][3]));
            }
            return most;
        };
        if (__any_sync(0xffffffffu, weigh() > M_MOST)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float top = fmaxf(x[t][i], x[t][i + 2]);
#pragma unroll
                    for (int b = 4; b < 32; b <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
                    const float to = top > m[t][i] + M_BELOW ? top - M_BELOW : m[t][i];
                    const float f = ex2(m[t][i] - to);
                    m[t][i] = to;
                    l[t][i] *= f;
#pragma unroll
                    for (int w = 0; w < DC; ++w) o[t][w][i] *= f, o[t][w][i + 2] *= f;
                }
            weigh();
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            l[t][0] = fmaf(p[t][0] + p[t][2], ivs, l[t][0]);
            l[t][1] = fmaf(p[t][1] + p[t][3], ivs, l[t][1]);
            const __half2 lo = __floats2half2_rn(p[t][0], p[t][1]), hi = __floats2half2_rn(p[t][2], p[t][3]);
            pb[t][0] = transpose8x8(*reinterpret_cast<const uint32_t *>(&lo));
            pb[t][1] = transpose8x8(*reinterpret_cast<const uint32_t *>(&hi));
        }
#pragma unroll
        for (int w = 0; w < DC; w += 2) {
            if (w >= nc) break;
            uint32_t r[4], f[4];
            ldsm4(va + w * 256, r);  // of an odd last chunk the second half is not used
            codes_a(r[0], r[1], f);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816(o[t][w], f, pb[t][0], pb[t][1]);
            if (w + 1 >= nc) break;
            codes_a(r[2], r[3], f);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816(o[t][w + 1], f, pb[t][0], pb[t][1]);
        }
    }

    __device__ __forceinline__ void close(int) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int b = 4; b < 32; b <<= 1) l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], b);
    }
    __device__ __forceinline__ void put(const KvAttnArgs &a, float *dst, int lane) const {
        const int g = lane >> 2, c = lane & 3;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 8 * t + 2 * c + i;
                if (g == 0) dst[2 * r] = m[t][i], dst[2 * r + 1] = l[t][i];
#pragma unroll
                for (int w = 0; w < DC; ++w) {
                    if (!FULL && w >= a.d / KV_B) break;
                    dst[part_head<RT>() + r * a.d + 16 * w + g] = o[t][w][i];
                    dst[part_head<RT>() + r * a.d + 16 * w + g + 8] = o[t][w][i + 2];
                }
            }
    }
    __device__ __forceinline__ void finish(const KvAttnArgs &a, const Seq &s, int h, int r0, int lane) const {
        const int g = lane >> 2, c = lane & 3;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int rr = r0 + 8 * t + 2 * c + i;
                if (rr >= s.n * a.group) continue;
                const int64_t row = row_index(a, s, h, rr);
                const float inv = l[t][i] == 0.0f ? 0.0f : 1.0f / l[t][i];
                uint16_t *dst = static_cast<uint16_t *>(a.out) + row * a.d + g;
                const bool bf = a.dtype == SKM_DTYPE_BF16;
#pragma unroll
                for (int w = 0; w < DC; ++w) {
                    if (!FULL && w >= a.d / KV_B) break;
                    dst[16 * w] = bits16(o[t][w][i] * inv, bf);
                    dst[16 * w + 8] = bits16(o[t][w][i + 2] * inv, bf);
                }
                if (g == 0 && a.lse) a.lse[row] = l[t][i] == 0.0f ? -INFINITY : LN2 * (m[t][i] + log2f(l[t][i]));
            }
    }
};

// A CTA's records of the units that its warps did not finish alone, in the
// line's order: [2 w] the unit that warp w found begun and left (part_warp), [2 w +
// 1] the one open at its end.
struct Record {
    int seq, unit;  // unit -1: none
    float *part;
};

// Shared memory of a CTA
struct Smem {
    size_t cum, seq, rec, win, bars, scratch, ring, warp_ring, total;
};
template <class Rows>
__host__ __device__ __forceinline__ constexpr Smem smem_of(int nb, int d, int nw, int ns) {
    Smem s = {};
    s.seq = s.cum + 8 * (size_t)(nb + 1);
    s.seq = (s.seq + 15) & ~size_t(15);
    s.rec = (s.seq + sizeof(Seq) * nb + 15) & ~size_t(15);
    s.win = s.rec + sizeof(Record) * 2 * nw;
    s.bars = s.win + sizeof(float4) * 64 * nw;
    s.scratch = (s.bars + 8 * (size_t)nw * ns + 127) & ~size_t(127);
    s.ring = (s.scratch + nw * Rows::scratch(d) + 127) & ~size_t(127);
    // a warp's ring, and after the loop its part of the unit still open
    const size_t ring = (size_t)ns * 2 * KV_B * d, part = (size_t)part_floats<Rows::RT>(d) * 4;
    s.warp_ring = ((ring > part ? ring : part) + 127) & ~size_t(127);
    s.total = s.ring + nw * s.warp_ring + 256;  // ldmatrix reads chunks in pairs
    return s;
}

__device__ __forceinline__ int64_t scan_add(int64_t x, int lane) {  // inclusive, over a warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// cum and seq of the launch's sequences (one sequence with `whole`); ends with
// a barrier
template <int RT>
__device__ void line_up(const KvAttnArgs &a, int b0, int nb, int64_t *cum, Seq *seq) {
    __shared__ int64_t warp_sum[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5;
    const auto items = [&](int i) {
        if (i >= nb) return int64_t(0);
        const Seq s = seq_of(a, b0 + i);
        seq[i] = s;
        return (int64_t)s.cnt * tiles_of(a, s, RT) * a.heads;
    };
    if (nb <= 32) {
        if (warp == 0) {
            const int64_t v = items(lane), x = scan_add(v, lane);
            if (lane < nb) cum[lane] = x - v;
            if (lane == 31) cum[nb] = x;
        }
        __syncthreads();
        return;
    }
    int64_t before = 0;
    for (int base = 0; base < nb; base += blockDim.x) {
        const int i = base + tid;
        const int64_t v = items(i), x = scan_add(v, lane);
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        const int64_t sums = scan_add(lane < nw ? warp_sum[lane] : 0, lane);
        const int64_t mine = warp ? __shfl_sync(0xffffffffu, sums, warp - 1) : 0;
        if (i < nb) cum[i] = before + mine + x - v;
        before += __shfl_sync(0xffffffffu, sums, 31);
        __syncthreads();
    }
    if (tid == 0) cum[nb] = before;
    __syncthreads();
}

// What the CTA that goes on with a unit first leaves for kv_join_kernel: the unit,
// the CTAs that hold parts of it (0: not this CTA's to say), its sequence's rows
struct Cut {
    int unit, parts, row0, n;
};
// The CTA that holds an item, C of them sharing W: CTA c takes [W c / C, W (c + 1) / C),
// with floor(W c / C) <= item written as W c < C (item + 1)
__device__ __forceinline__ int64_t holder(int64_t item, int64_t W, int64_t C) {
    int64_t c = (int64_t)((uint64_t)item * (uint64_t)C / (uint64_t)W);
    while (W * (c + 1) < C * (item + 1)) ++c;
    while (W * c >= C * (item + 1)) --c;
    return c;
}

// What this CTA (not the first) says of the unit [u0, u1) of W items that it found begun: parts 0 where
// another CTA was the first to go on with it
__device__ __forceinline__ Cut cut_of(int unit, const Seq &s, int64_t u0, int64_t u1, int64_t W, int64_t C) {
    const int64_t c = blockIdx.x;
    if (u0 < W * (c - 1) / C) return Cut{0, 0, 0, 0};
    return Cut{unit, (int)(holder(u1 - 1, W, C) - c + 2), s.row0, s.n};
}
// part_cta: [grid][2] parts (of the unit that the CTA found begun, of the one open at its end), [grid] Cuts
template <int RT>
__device__ __forceinline__ float *part_of(const KvAttnArgs &a, bool begun) {
    return a.part_cta + ((int64_t)blockIdx.x * 2 + (begun ? 0 : 1)) * part_floats<RT>(a.d);
}
template <int RT>
__device__ __forceinline__ Cut *cuts_of(const KvAttnArgs &a, int ctas) {
    return reinterpret_cast<Cut *>(a.part_cta + (int64_t)ctas * 2 * part_floats<RT>(a.d));
}

// A CTA of which a warp gave up its wait: that warp left items undone without a record, so all units of
// the CTA's stretch [c0, c1) become NaN, those shared with other CTAs by a part whose l is NaN.
template <int RT>
__device__ __noinline__ void give_up(const KvAttnArgs &a, Line line, int64_t c0, int64_t c1) {
    const int tid = threadIdx.x, n = blockDim.x;
    const int64_t W = line.cum[line.nb];
    if (tid == 0) {
        if (a.status) *a.status = 1;
        if (!a.whole) cuts_of<RT>(a, gridDim.x)[blockIdx.x] = Cut{0, 0, 0, 0};
    }
    for (int64_t item = c0; item < c1;) {
        const int b = line.find(item);
        const Seq s = line.seq[b];
        const int unit = (int)((item - line.cum[b]) / s.cnt);
        const int64_t u0 = line.cum[b] + (int64_t)unit * s.cnt, u1 = u0 + s.cnt;
        const int h = a.by_heads.mod(unit), r0 = a.by_heads.div(unit) * RT, rows = min(RT, s.n * a.group - r0);
        const bool all = u0 >= c0 && u1 <= c1;
        for (int r = tid; r < rows; r += n) {
            if (all) {
                const int64_t row = row_index(a, s, h, r0 + r);
                for (int i = 0; i < a.d; ++i) kv_store(a.out, row * a.d + i, NAN, a.dtype);
                if (a.lse) a.lse[row] = NAN;
            } else {
                float *part = part_of<RT>(a, u0 < c0);
                part[2 * r] = M_NONE, part[2 * r + 1] = NAN;
            }
        }
        if (tid == 0 && u0 < c0) cuts_of<RT>(a, gridDim.x)[blockIdx.x] = cut_of(unit, s, u0, u1, W, active_ctas(W, n / 32, gridDim.x));
        item = u1;
    }
}

template <class Rows, int NW>
__global__ void __launch_bounds__(NW * 32, 1) kv_rows_kernel(const __grid_constant__ KvAttnArgs a, int ns) {
    constexpr int RT = Rows::RT;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int gave_up;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // the sequences this CTA looks at, and its stretch of their line
    int nb = a.nb, b0 = a.b0, whole_unit = 0;
    if (a.whole) {
        const int per = a.max_tiles * a.heads;
        b0 += blockIdx.x / per;
        whole_unit = blockIdx.x % per;
        nb = 1;
    }
    const Smem sm = smem_of<Rows>(nb, a.d, NW, ns);
    int64_t *cum = reinterpret_cast<int64_t *>(smem + sm.cum);
    Seq *seq = reinterpret_cast<Seq *>(smem + sm.seq);
    Record *rec = reinterpret_cast<Record *>(smem + sm.rec);
    const uint32_t bars = su32(smem + sm.bars) + 8 * warp * ns;
    uint8_t *scratch = smem + sm.scratch + warp * Rows::scratch(a.d);
    const int half = KV_B * a.d;  // bytes of a block's keys
    uint8_t *ring = smem + sm.ring + warp * sm.warp_ring;
    const uint32_t ring_u = su32(ring);

    if (lane == 0)
        for (int i = 0; i < ns; ++i)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bars + 8 * i),
                         "r"(1 + (i == 0 && (int)blockIdx.x * NW + warp == a.stuck))
                         : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (lane < 2) rec[2 * warp + lane].unit = -1;
    if (tid == 0) gave_up = 0;
    line_up<RT>(a, b0, nb, cum, seq);
    const Line line{cum, seq, b0, nb};
    const int64_t W = cum[nb];
    int64_t c0, c1;  // this CTA's items
    if (a.whole) {
        const bool there = whole_unit < tiles_of(a, seq[0], RT) * a.heads;
        c0 = there ? (int64_t)whole_unit * seq[0].cnt : 0;
        c1 = there ? c0 + seq[0].cnt : 0;
    } else {
        const int64_t C = active_ctas(W, NW, gridDim.x), c = blockIdx.x;
        c0 = c < C ? W * c / C : 0;
        c1 = c < C ? W * (c + 1) / C : 0;
    }
    // rows of sequences without items: no key to see
    for (int i = a.whole ? 0 : blockIdx.x; i < nb; i += a.whole ? 1 : gridDim.x) {
        const Seq s = seq[i];
        if (s.cnt > 0 || s.n == 0 || (a.whole && whole_unit != 0)) continue;
        const int64_t row = s.row0, hq = a.heads * a.group;
        for (int64_t e = tid; e < s.n * hq * a.d; e += NW * 32) kv_store(a.out, row * hq * a.d + e, 0.0f, a.dtype);
        if (a.lse)
            for (int64_t e = tid; e < s.n * hq; e += NW * 32) a.lse[row * hq + e] = -INFINITY;
    }

    const int64_t i0 = c0 + (c1 - c0) * warp / NW, i1 = c0 + (c1 - c0) * (warp + 1) / NW;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the join waits for this kernel's end all the same
    Rows rows;
    bool open = false, ok = true;
    int useq = 0, uunit = 0;       // the open unit
    int ur0 = 0;                   // ... its first row of its sequence's
    int ublk = 0;                  // ... the block of the window's item 0, were it of this unit
    int safe_last = 0, safe_first = 0;  // blocks within [first, last] need no mask
    if (i1 > i0) {
        float4 *win = reinterpret_cast<float4 *>(smem + sm.win) + 64 * warp;
        int side = 0;  // half of win that holds cur's scales
        Window cur, next;
        window_pages<RT>(a, line, i0, i1, lane, cur);
        window_blocks(a, cur);
        int64_t base = i0;
        uint32_t to_issue = cur.todo, flying = 0;
        bool ahead = false, known = false;  // to_issue belongs to `next`; next's blocks are known
        int put_at = 0, take_at = 0;
        uint32_t phase = 0;  // parity of the stage taken next
        const auto issue = [&](int at) {
            if (lane == 0) {
                const uint32_t b = bars + 8 * put_at, dst = ring_u + put_at * 2 * half;
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(2u * half) : "memory");
                bulk_g2s(dst, a.k + (int64_t)at * half, half, b);
                bulk_g2s(dst + half, a.v + (int64_t)at * half, half, b);
            }
            put_at = put_at + 1 == ns ? 0 : put_at + 1;
            ++flying;
        };
        while (to_issue && flying < (uint32_t)ns) {  // the first copies go out before the next window is known
            const int i = __ffs(to_issue) - 1;
            to_issue &= to_issue - 1;
            issue(__shfl_sync(0xffffffffu, cur.at, i));
        }
        const auto fill_ring = [&] {
            while (flying < (uint32_t)ns) {
                if (!to_issue) {
                    if (ahead || !known) break;
                    ahead = true;
                    to_issue = next.todo;
                    continue;
                }
                const int i = __ffs(to_issue) - 1;
                to_issue &= to_issue - 1;
                issue(__shfl_sync(0xffffffffu, ahead ? next.at : cur.at, i));
            }
        };
        window_pages<RT>(a, line, base + 32, i1, lane, next);
        window_scales(cur, win, lane);
        const auto leave = [&](bool last) {  // the open unit ends here, for this warp
            const Seq s = seq[useq];
            rows.close(lane);
            const int64_t u0 = cum[useq] + (int64_t)uunit * s.cnt;
            const bool done = u0 >= i0 && u0 + s.cnt <= i1;
            if (done) {
                rows.finish(a, s, a.by_heads.mod(uunit), ur0, lane);
            } else if (!last) {
                float *dst = a.part_warp + ((int64_t)blockIdx.x * NW + warp) * part_floats<RT>(a.d);
                rows.put(a, dst, lane);
                if (lane == 0) rec[2 * warp] = Record{useq, uunit, dst};
            }
            return !done;
        };
        for (;;) {
            // next: its blocks a few items into this window, its scales some later
            for (int i = 0; i < cur.n; ++i) {
                if (i == 8) {
                    window_blocks(a, next);
                    known = true;
                    fill_ring();
                }
                if (i == 20) window_scales(next, win + 32 * (side ^ 1), lane);
                if (!open || ((cur.starts >> i) & 1)) {
                    if (open) leave(false);
                    open = true;
                    useq = __shfl_sync(0xffffffffu, cur.seq, i);
                    uunit = __shfl_sync(0xffffffffu, cur.unit, i);
                    ublk = __shfl_sync(0xffffffffu, cur.blk, i) - i;
                    const Seq s = seq[useq];
                    ur0 = a.by_heads.div(uunit) * RT;
                    safe_last = last_of(a, s, ur0);
                    safe_first = first_of(a, s, min(ur0 + RT, s.n * a.group) - 1);
                    rows.begin(a, s, a.by_heads.mod(uunit), ur0, scratch, lane);
                }
                if (!((cur.todo >> i) & 1)) continue;
                const int blk = ublk + i;
                const float4 sc = win[32 * side + i];
                if (!__all_sync(0xffffffffu, bar_wait(bars + 8 * take_at, phase, a.wait_ns))) {
                    ok = false;
                    break;
                }
                const uint8_t *K = ring + take_at * 2 * half;
                const bool mask = blk * KV_B < safe_first || blk * KV_B + KV_B - 1 > safe_last;
                rows.block(a, K, K + half, blk, sc.x, sc.y, sc.z, mask, lane);
                __syncwarp();
                if (++take_at == ns) take_at = 0, phase ^= 1u;
                --flying;
                fill_ring();
            }
            base += 32;
            if (base >= i1 || !ok) break;
            cur = next;
            side ^= 1;
            ublk += 32;
            if (ahead) ahead = false;
            else to_issue = cur.todo;
            known = false;
            window_pages<RT>(a, line, base + 32, i1, lane, next);
            fill_ring();
        }
        if (!ok) {  // a copy did not arrive: let the others land before the memory is given up
            for (; flying > 0; --flying) {
                bar_wait(bars + 8 * take_at, phase, a.wait_ns);
                if (++take_at == ns) take_at = 0, phase ^= 1u;
            }
            if (lane == 0) gave_up = 1;
        }
        open = ok && leave(true);
    }
    // a unit still open leaves its part where the warp's ring was
    const int64_t pf = part_floats<RT>(a.d);
    if (open) {
        float *dst = reinterpret_cast<float *>(ring);
        __syncwarp();
        rows.put(a, dst, lane);
        if (lane == 0) rec[2 * warp + 1] = Record{useq, uunit, dst};
    }
    __syncthreads();
    if (gave_up) {
        give_up<RT>(a, line, c0, c1);
        return;
    }
    const Record mine = lane < 2 * NW ? rec[lane] : Record{0, -1, nullptr};
    // (by a warp that has no rows to merge)
    Cut *cut = a.whole || warp != NW - 1 || lane != 0 ? nullptr : cuts_of<RT>(a, gridDim.x) + blockIdx.x;
    if (cut) *cut = Cut{0, 0, 0, 0};
    for (uint32_t left = __ballot_sync(0xffffffffu, mine.unit >= 0); left;) {
        const int f = __ffs(left) - 1;
        const int rs = __shfl_sync(0xffffffffu, mine.seq, f), ru = __shfl_sync(0xffffffffu, mine.unit, f);
        const uint32_t same = __ballot_sync(0xffffffffu, mine.unit == ru && mine.seq == rs);
        left &= ~same;
        const Seq s = seq[rs];
        const int64_t u0 = cum[rs] + (int64_t)ru * s.cnt, u1 = u0 + s.cnt;
        float *dst = u0 >= c0 && u1 <= c1 ? nullptr : part_of<RT>(a, u0 < c0);
        if (cut && u0 < c0) *cut = cut_of(ru, s, u0, u1, W, active_ctas(W, NW, gridDim.x));
        merge_parts<RT, Rows::D4>(a, mine.part, same, s, ru, dst, warp, NW, lane);
    }
}

// CTA c RT + r: row r of the unit that kv_rows_kernel's CTA c was the first to go on
// with; merges what the CTAs left of it, a warp every fourth part, then the warps' sums.
template <int RT>
__global__ void __launch_bounds__(128) kv_join_kernel(const __grid_constant__ KvAttnArgs a, int ctas) {
    __shared__ float tops[4], sl[4];
    __shared__ float2 ml[KV_SMS];  // (m, l) of the parts, then (weight, .)
    __shared__ float4 so[3][64];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = blockIdx.x % RT, c = blockIdx.x / RT;
    const int64_t pf = part_floats<RT>(a.d);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Cut cut = cuts_of<RT>(a, ctas)[c];
    const int unit = cut.unit, np = cut.parts;
    if (np == 0 || a.by_heads.div(unit) * RT + r >= cut.n * a.group) return;
    Seq s = {};
    s.row0 = cut.row0;
    // the CTA before left it open at its end (slot 1), this one and others found it begun (slot 0)
    const float *base = a.part_cta + (int64_t)(c - 1) * 2 * pf;
    const auto part = [&](int i) { return base + (2 * (int64_t)i + (i == 0 ? 1 : 0)) * pf; };
    float m = M_NONE;
    for (int i = tid; i < np; i += 128) {
        const float2 x = *reinterpret_cast<const float2 *>(part(i) + 2 * r);
        ml[i] = x;
        m = fmaxf(m, x.x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) tops[warp] = m;
    __syncthreads();
    m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    float l = 0.0f;
    for (int i = tid; i < np; i += 128) {
        const float f = ex2(ml[i].x - m);
        l = fmaf(ml[i].y, f, l);
        ml[i].x = f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) sl[warp] = l;
    __syncthreads();
    l = sl[0] + sl[1] + sl[2] + sl[3];
    float4 o[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
    const int d4 = a.d / 4;
#pragma unroll 4
    for (int i = warp; i < np; i += 4) {
        const float f = ml[i].x;
        const float4 *p = reinterpret_cast<const float4 *>(part(i) + part_head<RT>() + r * a.d);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (lane + 32 * k < d4) {
                const float4 v = p[lane + 32 * k];
                o[k].x = fmaf(v.x, f, o[k].x), o[k].y = fmaf(v.y, f, o[k].y);
                o[k].z = fmaf(v.z, f, o[k].z), o[k].w = fmaf(v.w, f, o[k].w);
            }
    }
    if (warp > 0)
        for (int k = 0; k < 2; ++k) so[warp - 1][lane + 32 * k] = o[k];
    __syncthreads();
    if (warp > 0) return;
    const int64_t row = row_index(a, s, a.by_heads.mod(unit),
                                  a.by_heads.div(unit) * RT + r);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    for (int k = 0; k < 2; ++k)
        if (lane + 32 * k < d4) {
            float4 v = o[k];
            for (int w = 0; w < 3; ++w) {
                const float4 x = so[w][lane + 32 * k];
                v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
            }
            store_row4(a, row, lane + 32 * k, v, inv);
        }
    if (lane == 0 && a.lse) a.lse[row] = l == 0.0f ? -INFINITY : LN2 * (m + log2f(l));
}

constexpr size_t SMEM_MOST = 226 * 1024;  // the static part aside

template <class Rows, int NW>
cudaError_t run_rows(const KvAttnArgs &a, const KvRowsPlan &p, cudaStream_t st) {
    static SmemLimit limit;
    cudaError_t e = limit.launch(kv_rows_kernel<Rows, NW>, SMEM_MOST, [&] {
        kv_rows_kernel<Rows, NW><<<(unsigned)p.grid, NW * 32, p.smem, st>>>(a, p.ns);
    });
    if (e != cudaSuccess || p.whole) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.grid * Rows::RT));
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kv_join_kernel<Rows::RT>, a, (int)p.grid);
    return e != cudaSuccess ? e : launched();
}

// One CTA a unit, without the join kernel: where every unit has an SM, and none is so
// long that it had better be shared.  16-bit queries, 4 heads a group, d = 128
// (alone in a graph): 8 units of 121 keys take 8 us against 12 in shared stretches,
// of 1001 both 12, of 1901 16 against 14; 128 units of 1901 17 against 20; 512 units of 121
// keys, more than a wave, 28 against 13, 192 of 1001 23 against 19.
constexpr int64_t WHOLE_FEW = 64, WHOLE_KEYS = 1024, WHOLE_KEYS_MANY = 2048;
bool whole_units(int64_t units, int64_t span) {
    return units <= KV_SMS && span <= (units <= WHOLE_FEW ? WHOLE_KEYS : WHOLE_KEYS_MANY);
}

// Sequences of one launch: their line takes 28 bytes of shared memory each, which 1024 of them have
// beside the smaller tiles only (32 rows of d = 128: 783; 16 of 256: 856)
template <class Rows>
int seqs_that_fit(int nb, int d, int nw) {
    nb = std::min(nb, KV_MAX_SEQS);
    while (smem_of<Rows>(nb, d, nw, 1).total > SMEM_MOST) --nb;  // (ends: plan_rows' assertion)
    return nb;
}

template <class Rows, int NW, int DMAX>
KvRowsPlan plan_rows(int nb, int heads, int group, int d, int max_tokens, int64_t span) {
    static_assert(smem_of<Rows>(1, DMAX, NW, 1).total <= SMEM_MOST, "a CTA's shared memory");
    constexpr int nw = NW;
    KvRowsPlan p = {};
    p.rt = Rows::RT;
    p.nw = nw;
    p.seqs = nb = seqs_that_fit<Rows>(nb, d, nw);
    p.units = (int64_t)nb * cdiv((int64_t)max_tokens * group, p.rt) * heads;
    p.whole = whole_units(p.units, span);
    p.ns = 4;
    const int seqs = p.whole ? 1 : nb;
    while (p.ns > 1 && smem_of<Rows>(seqs, d, nw, p.ns).total > SMEM_MOST) --p.ns;
    p.smem = smem_of<Rows>(seqs, d, nw, p.ns).total;
    p.grid = p.whole ? p.units : KV_SMS;
    p.part_cta = p.whole ? 0 : (size_t)p.grid * (2 * part_floats<Rows::RT>(d) * 4 + sizeof(Cut));
    p.part_warp = p.whole ? 0 : (size_t)p.grid * nw * part_floats<Rows::RT>(d) * 4;
    return p;
}

}  // namespace

// The variants.  fp32 queries: one row or four.  16-bit queries: tiles of 8,
// 16 or 32 rows (d > 128: 8 or 16, the sums of a tile are held in registers);
// warps as many as the registers of that tile allow.  A variant for d = 64, 128 or
// 256 only (FULL) has no bounds on dims in its loops, the other takes any d.
#define KV_ROWS_VARIANTS(X)                                                                              \
    X(1, 1, 64, (Fp32Rows<1, 2>), 16) X(1, 1, 128, (Fp32Rows<1, 4>), 16) X(1, 1, 256, (Fp32Rows<1, 8>), 8)  \
    X(1, 4, 64, (Fp32Rows<4, 2>), 16) X(1, 4, 128, (Fp32Rows<4, 4>), 16) X(1, 4, 256, (Fp32Rows<4, 8>), 8)  \
    KV_MMA_VARIANTS(X, true) KV_MMA_VARIANTS(X, false)
#define KV_MMA_VARIANTS(X, FULL)                                                                            \
    X(0, 8, 64, (MmaRows<4, 1, FULL>), 16) X(0, 8, 128, (MmaRows<8, 1, FULL>), 16)                          \
    X(0, 8, 256, (MmaRows<16, 1, FULL>), 8) X(0, 16, 64, (MmaRows<4, 2, FULL>), 16)                         \
    X(0, 16, 128, (MmaRows<8, 2, FULL>), 8) X(0, 16, 256, (MmaRows<16, 2, FULL>), 8)                        \
    X(0, 32, 64, (MmaRows<4, 4, FULL>), 8) X(0, 32, 128, (MmaRows<8, 4, FULL>), 8)

#define KV_UNPACK(...) __VA_ARGS__

// variants for one d only come before those that take any
template <class Rows>
constexpr bool is_full() {
    return Rows::ONE_D;
}

// span: positions that a unit's items may cover
KvRowsPlan kv_rows_plan(int nb, int heads, int group, int d, int dtype, int max_tokens, int64_t span) {
    const int64_t rows = (int64_t)max_tokens * group;
    const int fp32 = dtype == SKM_DTYPE_F32;
    const int rt = fp32 ? (rows == 1 ? 1 : 4) : (rows <= 8 ? 8 : rows <= 16 || d > 128 ? 16 : 32);
    const int dmax = d <= 64 ? 64 : d <= 128 ? 128 : 256;
#define KV_PLAN(FP32, RT, D, ROWS, NW)                                                          \
    if (fp32 == FP32 && rt == RT && dmax == D) {                                                \
        KvRowsPlan p = plan_rows<KV_UNPACK ROWS, NW, D>(nb, heads, group, d, max_tokens, span); \
        p.fp32 = FP32;                                                                          \
        return p;                                                                               \
    }
    KV_ROWS_VARIANTS(KV_PLAN)
#undef KV_PLAN
    return KvRowsPlan{};
}

size_t kv_rows_part_most(int nb, int heads, int d, int dtype, int64_t rows, int64_t span) {
    // fewer units may share an SM's stretch where more have one each
    if (span <= WHOLE_KEYS && (int64_t)nb * heads * cdiv(rows, (int64_t)(dtype == SKM_DTYPE_F32 ? 4 : 8)) <= KV_SMS) return 0;
    size_t most = 0;
    for (const int r : {1, 2, 9, 17}) {  // the fewest rows of every tile
        if (r > rows) break;
        const KvRowsPlan p = kv_rows_plan(KV_SMS + 1, 1, 1, d, dtype, r, WHOLE_KEYS_MANY + 1);
        Carver cv(nullptr, 0);
        cv.take<float>(p.part_cta / 4);
        cv.take<float>(p.part_warp / 4);
        most = std::max(most, cv.off);
    }
    return most;
}

cudaError_t launch_kv_rows(const KvAttnArgs &a, const KvRowsPlan &p, cudaStream_t st) {
    const int dmax = a.d <= 64 ? 64 : a.d <= 128 ? 128 : 256;
    const bool full = a.d == dmax;
#define KV_RUN(FP32, RT, D, ROWS, NW) \
    if (p.fp32 == FP32 && p.rt == RT && dmax == D && (full || !is_full<KV_UNPACK ROWS>())) \
        return run_rows<KV_UNPACK ROWS, NW>(a, p, st);
    KV_ROWS_VARIANTS(KV_RUN)
#undef KV_RUN
    return cudaErrorInvalidValue;
}

}  // namespace skm
