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
#include "skm_kv_rows.cuh"

namespace skm {

namespace {

// Rows of one warp in fp32 on CUDA cores.  Scores: lane = (half, token), a
// half takes every other 16-dim chunk of the keys; sums: lane = dims lane,
// lane + 32, ...  q and p pass through the warp's shared memory.
template <int R, int DPL>
struct Fp32Rows {
    static constexpr int RT = R, D4 = DPL > 4 ? 2 : 1;
    static constexpr bool ONE_D = false, FOUR = false;
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
    static constexpr bool ONE_D = FULL, FOUR = false;
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
    return rows_part_most(kv_rows_plan, nb, heads, d, dtype, rows, span);
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
