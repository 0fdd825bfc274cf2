// Attention over the 4-bit cache for few query rows (single tokens, a few
// tokens).  The line of blocks, its rings of bulk copies and its joining are those of
// k_kv_rows.cu (skm_kv_rows.cuh); a block is one copy here, its scales and biases included.
//
// Mathematics.  A token's key is b_k + s_k c, c its codes 0..15, so
//   S = scale log2(e) <q, k> = (scale log2(e) s_k) <q, c> + (scale log2(e) sum q) b_k,
// its value b_v + s_v c, so with weights e = 2^(S - m)
//   o = sum e s_v c + sum e b_v,   l = sum e:
// the codes are multiplied as they are, scales and biases cost a few operations a
// token and row.  In the 16-bit form the value scale enters the logits as log2 s_v (as in
// k_kv_rows.cu: the weights that become f16 then are p = e s_v, kept below 2^15 by the
// reference m), l = sum p / s_v and the biases' sum is sum p (b_v / s_v), in fp32.
//
// The second product has codes less 7.5 (and b_v / s_v + 7.5): the weights' rounding is an error of the codes' size.  Tensor
// cores cut a sum off towards 0 at every product, by some 2^-20 of it, so an item's products start from 0 and are added to the
// rows' sums in fp32 with rounding: a sum that every product of a stretch goes into loses 2^-20 of itself every 16 tokens, and with
// codes 0..15 the mean of a million values that nearly cancel was 2.7e-3 off where it is 2.0e-3 (codes less 8: 3.1e-5).
// For f16 outputs weights are two f16, a second product with the same codes: with one they are 1.1 to 1.56 times as far off an
// exact result as their rounding (60 cases of any sizes), with two 1.00 times.  bf16 outputs hide the rounding of one (1.01 times).
//
// A key's code as an operand of the tensor cores costs half an instruction: four bits under a mask
// are the f16 numbers 2^-24 c (bits 0..3) or 2^-20 c (bits 4..7), subnormal and
// exact, so a word's eight codes are four operands after one shift and four masks.  The factor
// 16 between the two lies on the other operand (half of a query's dims carry 2^-4), 2^24 on the
// results.  A logit has at most 16 such products.
//
// What bounds it, with a batch that fills the machine: the latencies of four warps a scheduler before HBM.
// 96 sequences of up to 10001 tokens, 8 heads of 128 dims, 4 query rows each, bf16: 124 us, 65% of a
// copy's rate (79.9 us for the bytes), 119 with codes 0..15 summed without a rounding.  bf16 and f16 are kernels of their own: in one, the
// second weights' registers cost bf16 calls 2 to 10% (20 rows 73 us, 66 now).  Items of two blocks share masks, maxima and the walk (138 -> 129 us), queries'
// operands lie in shared memory where registers would spill (129 -> 118).  A long sequence, f16, 262151 tokens: 74 us (42.2), with weights
// in one f16 66.
#include "skm_kv_rows.cuh"

namespace skm {

namespace {

// the scale and bias of a token's key and value, f16 x 4
struct TokenScales {
    float ks, kb, vs, vb;
};
__device__ __forceinline__ TokenScales token_scales(const uint8_t *rec, int d, int t) {
    const uint2 w = *reinterpret_cast<const uint2 *>(rec + KV_B * d + 8 * t);
    const float2 k = __half22float2(*reinterpret_cast<const __half2 *>(&w.x)), v = __half22float2(*reinterpret_cast<const __half2 *>(&w.y));
    return TokenScales{k.x, k.y, v.x, v.y};
}

constexpr float MIDDLE = 8.0f;
// the code in bits 0..3, less 8
__device__ __forceinline__ float code(uint32_t u) { return __uint_as_float((u & 15u) | 0x4b000000u) - (8388608.0f + MIDDLE); }

// Rows of one warp in fp32 on CUDA cores.  Scores: lane = (half, token), a half takes every
// other 16-dim chunk of the keys; sums: lane = dims lane, lane + 32, ...  q and the
// weights pass through the warp's shared memory.
template <int R, int DPL>
struct Fp32Rows4 {
    static constexpr int RT = R, D4 = DPL > 4 ? 2 : 1;
    static constexpr bool ONE_D = false, FOUR = true, HALF = false;
    static constexpr size_t __host__ __device__ scratch(int d) { return (size_t)R * (d + KV_B) * 4 + LIMITS<R>; }
    float o[R][DPL], m[R], l[R], ob[R], qs[R];  // ob: the biases' sum, qs: the query's
    float *q, *p;
    int2 *lim;

    __device__ __forceinline__ void begin(const KvAttnArgs &a, const Seq &s, int h, int r0, uint8_t *mem, int lane) {
        lim = reinterpret_cast<int2 *>(mem);
        q = reinterpret_cast<float *>(mem + LIMITS<R>);
        p = q + R * a.d;
        __syncwarp();
        limits<R>(a, s, r0, lim, lane);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = M_NONE, l[r] = ob[r] = qs[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < DPL; ++i) o[r][i] = 0.0f;
            const int rr = r0 + r;
            const bool in = rr < s.n * a.group;
            const int64_t at = in ? (int64_t)(s.row0 + a.by_group.div(rr)) * a.q_token + (int64_t)(h * a.group + a.by_group.mod(rr)) * a.q_head : 0;
            for (int i = lane; i < a.d; i += 32) {
                const float x = in ? kv_load(a.Q, at + i, a.dtype) * a.scale_log2 : 0.0f;
                q[r * a.d + i] = x;
                qs[r] += x;
            }
#pragma unroll
            for (int b = 16; b > 0; b >>= 1) qs[r] += __shfl_xor_sync(0xffffffffu, qs[r], b);
        }
        __syncwarp();
    }

    __device__ __forceinline__ void item(const KvAttnArgs &a, const uint8_t *rec, int pair, bool mask, uint32_t have, int lane) {
#pragma unroll 1
        for (int i = 0; i < 2; ++i)
            if (have >> i & 1) block(a, rec + i * kv4_bytes(a.d), 2 * pair + i, mask, lane);
    }
    __device__ __forceinline__ void block(const KvAttnArgs &a, const uint8_t *rec, int blk, bool mask, int lane) {
        const int t = lane & 15, half = lane >> 4, nc = a.d / KV_B;
        const uint8_t *K = rec, *V = rec + 8 * a.d;
        TokenScales sc = token_scales(rec, a.d, t);
        sc.kb = fmaf(MIDDLE, sc.ks, sc.kb), sc.vb = fmaf(MIDDLE, sc.vs, sc.vb);  // codes around their middle: smaller sums
        float x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = 0.0f;
        for (int w = half; w < nc; w += 2) {
            const uint4 c = *reinterpret_cast<const uint4 *>(K + w * 128 + (t & 7) * 16);
            const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u = word[i] >> (t & 8);  // codes of the token's dims 4 i, + 2, . , . , + 1, + 3
                const float k0 = code(u), k2 = code(u >> 4), k1 = code(u >> 16), k3 = code(u >> 20);
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
        bool seen = !mask;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            x[r] += __shfl_xor_sync(0xffffffffu, x[r], 16);
            x[r] = fmaf(x[r], sc.ks, qs[r] * sc.kb);
            if (mask) {
                const int j = blk * KV_B + t;
                if (j > lim[r].x || j < lim[r].y) x[r] = -INFINITY;
                else seen = true;
            }
            if (__any_sync(0xffffffffu, x[r] > m[r] + M_SLACK)) {
                float top = x[r];
#pragma unroll
                for (int b = 8; b > 0; b >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
                const float to = top - M_BELOW, f = exp2f(m[r] - to);
                m[r] = to;
                l[r] *= f;
                ob[r] *= f;
#pragma unroll
                for (int i = 0; i < DPL; ++i) o[r][i] *= f;
            }
        }
        if (!seen) sc.vs = sc.vb = 0.0f;  // (a token that was never written has no scales)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float e = exp2f(x[r] - m[r]);
            if (half == 0) {
                l[r] += e;
                ob[r] = fmaf(e, sc.vb, ob[r]);
                p[r * KV_B + t] = e * sc.vs;
            }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            const int dim = lane + 32 * i;
            if (dim >= a.d) break;
            const uint4 c = *reinterpret_cast<const uint4 *>(V + (dim >> 4) * 128 + (dim & 7) * 16);
            const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t u = word[w] >> (dim & 8);  // codes of tokens 2 w, + 8, . , . , + 1, + 9
                const float v0 = code(u), v8 = code(u >> 4), v1 = code(u >> 16), v9 = code(u >> 20);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float2 lo = *reinterpret_cast<const float2 *>(p + r * KV_B + 2 * w);
                    const float2 hi = *reinterpret_cast<const float2 *>(p + r * KV_B + 2 * w + 8);
                    o[r][i] = fmaf(v0, lo.x, o[r][i]);
                    o[r][i] = fmaf(v1, lo.y, o[r][i]);
                    o[r][i] = fmaf(v8, hi.x, o[r][i]);
                    o[r][i] = fmaf(v9, hi.y, o[r][i]);
                }
            }
        }
        __syncwarp();
    }

    __device__ __forceinline__ void close(int) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int b = 16; b > 0; b >>= 1) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], b);
                ob[r] += __shfl_xor_sync(0xffffffffu, ob[r], b);
            }
#pragma unroll
            for (int i = 0; i < DPL; ++i) o[r][i] += ob[r];
        }
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

// the codes of a lane's word (rows g and g + 8 of a 16 x 16 tile, columns 2c, 2c + 1 and 2c + 8, 2c + 9) as
// operand A: 2^-24 times the first two columns', 2^-20 times the others'
__device__ __forceinline__ void codes4_a(uint32_t w, uint32_t (&a)[4]) {
    a[0] = w & 0x000f000fu;
    a[2] = w & 0x00f000f0u;
    w >>= 8;
    a[1] = w & 0x000f000fu;
    a[3] = w & 0x00f000f0u;
}
constexpr float CODES_UP = 16777216.0f;   // 2^24
// 2^-9 times the same codes less 7.5, exact: subnormal as they are, one fused multiply-add each
constexpr float CENTRE = 7.5f, CENTRED_UP = 512.0f;  // 2^9
__device__ __forceinline__ void codes4_centred(uint32_t w, uint32_t (&a)[4]) {
    const auto half2 = [](uint32_t x) { return *reinterpret_cast<const __half2 *>(&x); };
    const auto less = [&](uint32_t x, uint32_t up) {  // up: 2^15 or 2^11; 0xa380: -7.5 2^-9
        const __half2 r = __hfma2(half2(x), half2(up), half2(0xa380a380u));
        return *reinterpret_cast<const uint32_t *>(&r);
    };
    a[0] = less(w & 0x000f000fu, 0x78007800u), a[2] = less(w & 0x00f000f0u, 0x68006800u);
    w >>= 8;
    a[1] = less(w & 0x000f000fu, 0x78007800u), a[3] = less(w & 0x00f000f0u, 0x68006800u);
}
constexpr float SCALE_LEAST = 5.9604645e-8f;  // 2^-24, the smallest f16 above 0: a scale of 0 (then all codes are 0) counts as it

// Rows of one warp on tensor cores, transposed as in k_kv_rows.cu: S^T = K q^T and o^T =
// V^T p^T.  A lane's word of a chunk is a 16 x 16 operand's own eight codes; ldmatrix
// brings the words of four chunks.  Queries, of either type, become f16 after scaling a row by a power of two
// that takes its largest element to [2^15, 2^16) (to_f16), dims 4c + 2, 4c + 3 with 2^-4 on top: bf16
// elements down to 2^-28 of the row's largest and f16 ones down to 2^-25 take part exactly.
// DC: 16-dim chunks at most (FULL: exactly), NT: tiles of 8 rows, F16: queries and outputs are f16, else bf16.
template <int DC, int NT, bool FULL, bool F16>
struct MmaRows4 {
    static constexpr int RT = 8 * NT;
    static constexpr int D4 = DC > 8 ? 2 : 1;
    static constexpr bool ONE_D = FULL, FOUR = true, HALF = F16;
    static constexpr bool QMEM = NT * DC >= 8;  // the queries' operands wait in shared memory (decode batch 118 us, in registers 129)
    static constexpr size_t __host__ __device__ scratch(int) { return (QMEM ? (size_t)NT * DC * 2 * 32 * 4 : 0) + LIMITS<RT>; }
    float o[NT][DC][4], m[NT][2], l[NT][2], ob[NT][2], fac[NT][2], qs[NT][2];
    uint32_t q[QMEM ? 1 : NT][QMEM ? 1 : DC][2];
    uint2 *qmem;
    int2 *lim;

    __device__ __forceinline__ void begin(const KvAttnArgs &a, const Seq &s, int h, int r0, uint8_t *mem, int lane) {
        const int g = lane >> 2, c = lane & 3, nc = FULL ? DC : a.d / KV_B;
        lim = reinterpret_cast<int2 *>(mem);
        qmem = reinterpret_cast<uint2 *>(mem + LIMITS<RT>);
        __syncwarp();
        limits<RT>(a, s, r0, lim, lane);
        const auto pair = [&](uint32_t w) {
            if constexpr (!F16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
            else return __half22float2(*reinterpret_cast<const __half2 *>(&w));
        };
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
            uint32_t top = 0;  // the largest |x| as bits (of one sign, they order like the numbers)
#pragma unroll
            for (int w = 0; w < DC; ++w) {
                const float2 u = pair(raw[w].x), v = pair(raw[w].y);
                top = max(max(top, __float_as_uint(u.x) & 0x7fffffffu), __float_as_uint(u.y) & 0x7fffffffu);
                top = max(max(top, __float_as_uint(v.x) & 0x7fffffffu), __float_as_uint(v.y) & 0x7fffffffu);
            }
#pragma unroll
            for (int b = 1; b < 4; b <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, b));
            const Pow2 by = to_f16(top >> 23);
            float sum = 0.0f;
            const auto f16 = [&](float2 u, float less) {
                u.x *= by.mul, u.y *= by.mul;
                sum += u.x + u.y;
                const __half2 r = __floats2half2_rn(u.x * less, u.y * less);
                return *reinterpret_cast<const uint32_t *>(&r);
            };
#pragma unroll
            for (int w = 0; w < DC; ++w) {
                const uint32_t b0 = f16(pair(raw[w].x), 1.0f), b1 = f16(pair(raw[w].y), 0.0625f);
                if constexpr (QMEM) qmem[(t * DC + w) * 32 + lane] = make_uint2(b0, b1);
                else q[t][w][0] = b0, q[t][w][1] = b1;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[t][w][i] = 0.0f;
            }
            const float back = by.back * a.scale_log2;
#pragma unroll
            for (int b = 1; b < 4; b <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, b);
            sum *= back;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fac[t][i] = __shfl_sync(0xffffffffu, back, (2 * c + i) * 4);
                qs[t][i] = __shfl_sync(0xffffffffu, sum, (2 * c + i) * 4);
                m[t][i] = M_NONE;
                l[t][i] = ob[t][i] = 0.0f;
            }
        }
        __syncwarp();
    }

    // Two blocks at once where the rows are one tile: twice the independent products and half the tests of the
    // reference (decode batch below: 138 us with one at a time)
    __device__ __forceinline__ void item(const KvAttnArgs &a, const uint8_t *rec, int pair, bool mask, uint32_t have, int lane) {
        if (NT == 1 && have == 3) {
            blocks<2>(a, rec, 2 * pair, mask, lane);
            return;
        }
#pragma unroll 1
        for (int i = 0; i < 2; ++i)
            if (have >> i & 1) blocks<1>(a, rec + i * kv4_bytes(a.d), 2 * pair + i, mask, lane);
    }
    template <int NB>
    __device__ __forceinline__ void blocks(const KvAttnArgs &a, const uint8_t *rec, int blk, bool mask, int lane) {
        const int g = lane >> 2, c = lane & 3, nc = FULL ? DC : a.d / KV_B, bytes = kv4_bytes(FULL ? 16 * DC : a.d);
        float x[NB][NT][4];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[n][t][i] = 0.0f;
        const uint32_t ka = su32(rec) + lane * 16, va = ka + 8 * a.d;
#pragma unroll
        for (int w0 = 0; w0 < DC; w0 += 4) {
            if (w0 >= nc) break;
            uint32_t r[NB][4], f[4];
#pragma unroll
            for (int n = 0; n < NB; ++n) ldsm4(ka + n * bytes + w0 * 128, r[n]);  // (of the last chunks what lies behind them is not used)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int w = w0 + i;
                if (w >= DC || w >= nc) break;
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    codes4_a(r[n][i], f);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (QMEM) {
                            const uint2 b = qmem[(t * DC + w) * 32 + lane];
                            mma16816(x[n][t], f, b.x, b.y);
                        } else {
                            mma16816(x[n][t], f, q[t][w][0], q[t][w][1]);
                        }
                    }
                }
            }
        }
        // log2 and reciprocal of the value scales, biases over scales, of tokens g and g + 8
        float iv[NB][2], bv[NB][2];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const TokenScales sc = token_scales(rec + n * bytes, a.d, g + 8 * k);
                const float ks = sc.ks * CODES_UP, v = fmaxf(sc.vs, SCALE_LEAST);
                float lv;
                asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lv) : "f"(v));
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(iv[n][k]) : "f"(v));
                bv[n][k] = fmaf(sc.vb, iv[n][k], CENTRE);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        x[n][t][2 * k + i] = fmaf(x[n][t][2 * k + i], fac[t][i] * ks, fmaf(qs[t][i], sc.kb, lv));
            }
        if (mask) {
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                bool seen[2] = {false, false};
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = (blk + n) * KV_B + g + 8 * (i >> 1);
                        const int2 see = lim[8 * t + 2 * c + (i & 1)];
                        if (j > see.x || j < see.y) x[n][t][i] = -INFINITY;
                        else seen[i >> 1] = true;
                    }
                // a token that none of the lane's rows sees has no weight, but may never have been written
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (!seen[k]) iv[n][k] = bv[n][k] = 0.0f;
            }
        }
        float p[NB][NT][4];
        const auto weigh = [&] {  // weights, and the largest sum of two
            float most = 0.0f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[n][t][i] = ex2(x[n][t][i] - m[t][i & 1]);
                    most = fmaxf(most, fmaxf(p[n][t][0] + p[n][t][2], p[n][t][1] + p[n][t][3]));
                }
            return most;
        };
        if (__any_sync(0xffffffffu, weigh() > M_MOST)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float top = fmaxf(x[0][t][i], x[0][t][i + 2]);
#pragma unroll
                    for (int n = 1; n < NB; ++n) top = fmaxf(top, fmaxf(x[n][t][i], x[n][t][i + 2]));
#pragma unroll
                    for (int b = 4; b < 32; b <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
                    const float to = top > m[t][i] + M_BELOW ? top - M_BELOW : m[t][i];
                    const float f = ex2(m[t][i] - to);
                    m[t][i] = to;
                    l[t][i] *= f;
                    ob[t][i] *= f;
#pragma unroll
                    for (int w = 0; w < DC; ++w) o[t][w][i] *= f, o[t][w][i + 2] *= f;
                }
            weigh();
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    l[t][i] = fmaf(p[n][t][i + 2], iv[n][1], fmaf(p[n][t][i], iv[n][0], l[t][i]));
                    ob[t][i] = fmaf(p[n][t][i + 2], bv[n][1], fmaf(p[n][t][i], bv[n][0], ob[t][i]));
                }
        uint32_t pb[NB][NT][2];
        [[maybe_unused]] uint32_t pl[F16 ? NB : 1][NT][2];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float2 y = make_float2(p[n][t][2 * k], p[n][t][2 * k + 1]);
                    if constexpr (F16) {  // the upper part cut off, and what is left
                        const float2 z = make_float2(__uint_as_float(__float_as_uint(y.x) & 0xffffe000u), __uint_as_float(__float_as_uint(y.y) & 0xffffe000u));
                        const __half2 rest = __floats2half2_rn(y.x - z.x, y.y - z.y);
                        pl[n][t][k] = transpose8x8(*reinterpret_cast<const uint32_t *>(&rest));
                        y = z;
                    }
                    const __half2 w = __floats2half2_rn(y.x, y.y);
                    pb[n][t][k] = transpose8x8(*reinterpret_cast<const uint32_t *>(&w));
                }
#pragma unroll
        for (int w0 = 0; w0 < DC; w0 += 4) {
            if (w0 >= nc) break;
            uint32_t r[NB][4], f[4];
#pragma unroll
            for (int n = 0; n < NB; ++n) ldsm4(va + n * bytes + w0 * 128, r[n]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int w = w0 + i;
                if (w >= DC || w >= nc) break;
                float x[NT][4];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    codes4_centred(r[n][i], f);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if (n == 0) x[t][0] = x[t][1] = x[t][2] = x[t][3] = 0.0f;
                        mma16816(x[t], f, pb[n][t][0], pb[n][t][1]);
                        if constexpr (F16) mma16816(x[t], f, pl[n][t][0], pl[n][t][1]);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        const float2 y = add2(make_float2(o[t][w][k], o[t][w][k + 1]), make_float2(x[t][k], x[t][k + 1]));
                        o[t][w][k] = y.x, o[t][w][k + 1] = y.y;
                    }
            }
        }
    }

    __device__ __forceinline__ void close(int) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int b = 4; b < 32; b <<= 1) {
                    l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], b);
                    ob[t][i] += __shfl_xor_sync(0xffffffffu, ob[t][i], b);
                }
#pragma unroll
                for (int w = 0; w < DC; ++w) {
                    o[t][w][i] = fmaf(o[t][w][i], CENTRED_UP, ob[t][i]);
                    o[t][w][i + 2] = fmaf(o[t][w][i + 2], CENTRED_UP, ob[t][i]);
                }
            }
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
#pragma unroll
                for (int w = 0; w < DC; ++w) {
                    if (!FULL && w >= a.d / KV_B) break;
                    const float x = o[t][w][i] * inv, y = o[t][w][i + 2] * inv;
                    if constexpr (F16) {
                        const uint32_t u = kv_f16_within(x, y);
                        dst[16 * w] = (uint16_t)u, dst[16 * w + 8] = (uint16_t)(u >> 16);
                    } else {
                        dst[16 * w] = __bfloat16_as_ushort(__float2bfloat16_rn(x)), dst[16 * w + 8] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
                    }
                }
                if (g == 0 && a.lse) a.lse[row] = l[t][i] == 0.0f ? -INFINITY : LN2 * (m[t][i] + log2f(l[t][i]));
            }
    }
};

}  // namespace

// The variants: those of the 8-bit cache (k_kv_rows.cu)
#define KV4_ROWS_VARIANTS(X)                                                                                  \
    X(1, 1, 64, (Fp32Rows4<1, 2>), 16) X(1, 1, 128, (Fp32Rows4<1, 4>), 16) X(1, 1, 256, (Fp32Rows4<1, 8>), 8)  \
    X(1, 4, 64, (Fp32Rows4<4, 2>), 16) X(1, 4, 128, (Fp32Rows4<4, 4>), 16) X(1, 4, 256, (Fp32Rows4<4, 8>), 8)  \
    KV4_MMA_VARIANTS(X, true, false) KV4_MMA_VARIANTS(X, false, false) KV4_MMA_VARIANTS(X, true, true) KV4_MMA_VARIANTS(X, false, true)
#define KV4_MMA_VARIANTS(X, FULL, F16)                                                                        \
    X(0, 8, 64, (MmaRows4<4, 1, FULL, F16>), 16) X(0, 8, 128, (MmaRows4<8, 1, FULL, F16>), 16)                \
    X(0, 8, 256, (MmaRows4<16, 1, FULL, F16>), 8) X(0, 16, 64, (MmaRows4<4, 2, FULL, F16>), 16)               \
    X(0, 16, 128, (MmaRows4<8, 2, FULL, F16>), 8) X(0, 16, 256, (MmaRows4<16, 2, FULL, F16>), 8)              \
    X(0, 32, 64, (MmaRows4<4, 4, FULL, F16>), 8) X(0, 32, 128, (MmaRows4<8, 4, FULL, F16>), 8)

#define KV_UNPACK(...) __VA_ARGS__

KvRowsPlan kv4_rows_plan(int nb, int heads, int group, int d, int dtype, int max_tokens, int64_t span) {
    const int64_t rows = (int64_t)max_tokens * group;
    const int fp32 = dtype == SKM_DTYPE_F32;
    const int rt = fp32 ? (rows == 1 ? 1 : 4) : (rows <= 8 ? 8 : rows <= 16 || d > 128 ? 16 : 32);
    const int dmax = d <= 64 ? 64 : d <= 128 ? 128 : 256;
#define KV4_PLAN(FP32, RT, D, ROWS, NW)                                                         \
    if (fp32 == FP32 && rt == RT && dmax == D) {                                                \
        KvRowsPlan p = plan_rows<KV_UNPACK ROWS, NW, D>(nb, heads, group, d, max_tokens, span); \
        p.fp32 = FP32;                                                                          \
        return p;                                                                               \
    }
    KV4_ROWS_VARIANTS(KV4_PLAN)
#undef KV4_PLAN
    return KvRowsPlan{};
}

size_t kv4_rows_part_most(int nb, int heads, int d, int dtype, int64_t rows, int64_t span) {
    return rows_part_most(kv4_rows_plan, nb, heads, d, dtype, rows, span);
}

cudaError_t launch_kv4_rows(const KvAttnArgs &a, const KvRowsPlan &p, cudaStream_t st) {
    const int dmax = a.d <= 64 ? 64 : a.d <= 128 ? 128 : 256;
    const bool full = a.d == dmax, half = a.dtype == SKM_DTYPE_F16;
#define KV4_RUN(FP32, RT, D, ROWS, NW)                                                             \
    if (p.fp32 == FP32 && p.rt == RT && dmax == D && (full || !KV_UNPACK ROWS::ONE_D) && half == KV_UNPACK ROWS::HALF) \
        return run_rows<KV_UNPACK ROWS, NW>(a, p, st);
    KV4_ROWS_VARIANTS(KV4_RUN)
#undef KV4_RUN
    return cudaErrorInvalidValue;
}

}  // namespace skm
