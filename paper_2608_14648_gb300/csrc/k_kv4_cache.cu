// Writing keys and values into the 4-bit cache and reading them back.
//
// A token's key (or value) of a head is one LVQ vector: bias b, the largest f16 not above its
// smallest element, scale s, the smallest f16 with b + 15 s not below its largest, codes
// rint((x - b) / s).  One warp takes one block (16 tokens) of one head's keys or values and holds
// it in registers, so the input is read once: smallest and largest in registers and over a few lanes, then
// the codes.  A vector's codes depend on nothing else: what the block holds is never rounded again.
//
// Lanes.  Keys: (g, c), tokens g and g + 8, of every 32 dims the eight from 8 c on: a token's 32 dims
// are 64 consecutive bytes of 16-bit input, and the lane's codes are two neighbouring words.
// Values: (e, c), dims 8 e .. of the four tokens 2c, 2c + 1, 2c + 8, 2c + 9 that share a word; the
// other dims of a word are those of the lane next to it in e.
//
// Rounding.  q = (x - b) (1 / s) in fp32 takes three roundings of 2^-24 on the way to a number below
// 16, so it is within 3 2^-20 of the quotient, whose nearest integer is q's unless q lies within 2^-18 of
// the middle of two: then x - b is compared with (k + 1/2) s in 64 bits.
// Codes become words by multiply-adds of integers as floats (below 2^16, exact), two at a time.
#include "skm_kv_cache.cuh"

namespace skm {

namespace {

constexpr float MAGIC = 12582912.0f;  // 1.5 2^23: x + this, less this, is rint(x)
constexpr float NEAR = 0.5f - 3.8146973e-6f;  // 1/2 - 2^-18
constexpr float F16_MOST = 65504.0f;

// values 2 i and 2 i + 1 of words
template <typename T>
__device__ __forceinline__ float2 value2(const uint32_t *w, int i) {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2 *>(w + i));
    else return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}

// Smallest and largest of some values, NaN where one of them is
struct Range {
    float lo, hi;
};
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ Range both(Range a, Range b) { return Range{min_nan(a.lo, b.lo), max_nan(a.hi, b.hi)}; }
__device__ __forceinline__ Range across(Range r, int lanes) {
    return both(r, Range{__shfl_xor_sync(0xffffffffu, r.lo, lanes), __shfl_xor_sync(0xffffffffu, r.hi, lanes)});
}
// ... of 8 values
template <typename T>
__device__ __forceinline__ Range range8(const uint32_t *w) {
    if constexpr (std::is_same<T, float>::value) {
        Range r{__uint_as_float(w[0]), __uint_as_float(w[0])};
#pragma unroll
        for (int i = 1; i < 8; ++i) r = both(r, Range{__uint_as_float(w[i]), __uint_as_float(w[i])});
        return r;
    } else {
        using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        T2 lo = *reinterpret_cast<const T2 *>(w), hi = lo;
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            const T2 x = *reinterpret_cast<const T2 *>(w + i);
            lo = __hmin2_nan(lo, x);
            hi = __hmax2_nan(hi, x);
        }
        const uint32_t l = *reinterpret_cast<const uint32_t *>(&lo), h = *reinterpret_cast<const uint32_t *>(&hi);
        const float2 a = value2<T>(&l, 0), b = value2<T>(&h, 0);
        return Range{min_nan(a.x, a.y), max_nan(b.x, b.y)};
    }
}
__device__ __forceinline__ bool ordinary(Range r) { return r.lo >= -F16_MOST && r.hi <= F16_MOST; }

// Vectors that are not: the range of their finite elements, clipped to f16's
template <typename T>
__device__ __noinline__ float2 finite8(const uint32_t *w, float2 r) {
    for (int i = 0; i < 4; ++i) {
        const float2 p = value2<T>(w, i);
        if (fabsf(p.x) < INFINITY) r.x = fminf(r.x, p.x), r.y = fmaxf(r.y, p.x);
        if (fabsf(p.y) < INFINITY) r.x = fminf(r.x, p.y), r.y = fmaxf(r.y, p.y);
    }
    return r;
}
__device__ __forceinline__ Range clipped(float2 r) {
    if (r.x > r.y) return Range{0.0f, 0.0f};  // no finite element
    return Range{fminf(fmaxf(r.x, -F16_MOST), F16_MOST), fminf(fmaxf(r.y, -F16_MOST), F16_MOST)};
}

struct Lvq {
    float b, s, inv;
};
__device__ __forceinline__ Lvq lvq_of(Range r) {
    Lvq v;
    v.b = __half2float(__float2half_rd(r.lo));
    // three roundings upward: the scale wanted, or the f16 after it
    const uint16_t up = __half_as_ushort(__float2half_ru(__fdiv_ru(__fsub_ru(r.hi, v.b), 15.0f)));
    v.s = __half2float(__ushort_as_half(up));
    if (up) {
        const float less = __half2float(__ushort_as_half((uint16_t)(up - 1))), p = 15.0f * less;  // exact: 15 bits
        // b + p as an exact sum of two floats (Knuth, The Art of Computer Programming 2, 4.2.2), compared with hi
        const float sum = __fadd_rn(v.b, p), z = __fsub_rn(sum, v.b);
        const float err = __fadd_rn(__fsub_rn(v.b, __fsub_rn(sum, z)), __fsub_rn(p, z));
        if (__fadd_rn(__fsub_rn(sum, r.hi), err) >= 0.0f) v.s = less;
    }
    v.inv = v.s > 0.0f ? __frcp_rn(v.s) : 0.0f;
    return v;
}
__device__ __forceinline__ uint32_t held(const Lvq &v) {  // (scale, bias)
    const __half2 h = __floats2half2_rn(v.s, v.b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// the code of a value that fp32 leaves open, near the middle of two
__device__ __noinline__ float code_near(float x, float b, float s) {
    const float k = floorf((x - b) / s);
    const double over = (double)x - (double)b, mid = ((double)k + 0.5) * (double)s;
    return over > mid || (over == mid && ((int)k & 1)) ? k + 1.0f : k;
}
// codes of 8 values as floats
template <typename T>
__device__ __forceinline__ void codes8(const uint32_t *w, const Lvq &v, float2 *c) {
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 q = mul2(add2(value2<T>(w, i), make_float2(-v.b, -v.b)), make_float2(v.inv, v.inv));
        c[i] = add2(add2(q, make_float2(MAGIC, MAGIC)), make_float2(-MAGIC, -MAGIC));
        far = fmaxf(far, fmaxf(fabsf(q.x - c[i].x), fabsf(q.y - c[i].y)));
    }
    if (far > NEAR) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = value2<T>(w, i);
            if (fabsf((x.x - v.b) * v.inv - c[i].x) > NEAR) c[i].x = code_near(x.x, v.b, v.s);
            if (fabsf((x.y - v.b) * v.inv - c[i].y) > NEAR) c[i].y = code_near(x.y, v.b, v.s);
        }
    }
}
// ... of a vector that is not ordinary: its elements taken into its range, NaN to the smallest
template <typename T>
__device__ __noinline__ void codes8_clipped(const uint32_t *w, Lvq v, float lo, float hi, float2 *c) {
    for (int i = 0; i < 4; ++i) {
        const float2 p = value2<T>(w, i);
        float x[2] = {p.x, p.y};
        for (int k = 0; k < 2; ++k) {
            x[k] = x[k] == x[k] ? fminf(fmaxf(x[k], lo), hi) : lo;
            const float q = (x[k] - v.b) * v.inv, r = rintf(q);
            x[k] = fabsf(q - r) > NEAR ? code_near(x[k], v.b, v.s) : r;
        }
        c[i] = make_float2(x[0], x[1]);
    }
}

__device__ __forceinline__ float2 pack2(float2 a, float2 b, float up) { return fma2(b, make_float2(up, up), a); }
// two integers below 2^16 as the halves of a word
__device__ __forceinline__ uint32_t word_of(float lo, float hi) {
    return __byte_perm(__float_as_uint(lo + 8388608.0f), __float_as_uint(hi + 8388608.0f), 0x5410);
}
__device__ __forceinline__ uint32_t merged(uint32_t was, uint32_t now, uint32_t mask) { return (was & ~mask) | (now & mask); }

// Warps: one a (sequence, block its new rows reach, head, tensor).  D: dims at most
template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32) kv4_write_kernel(const __grid_constant__ KvCacheArgs a) {
    constexpr int W = WORDS8<T>;
    const int lane = threadIdx.x & 31;
    const int warp = blockIdx.x * WARPS + (threadIdx.x >> 5), tensor = warp & 1;
    const int h = a.by_heads.mod(warp >> 1);
    const Place at_block = place_of(a, a.by_heads.div(warp >> 1), lane);
    const int b = at_block.b;
    if (b >= a.batch) return;
    const int2 rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
    const int cap = a.cols * a.page;
    const int start = kv_clamp(a.pos[b], 0, cap);  // (from cap on there is nothing, and block positions stay below 2^31)
    const int end = (int)min((int64_t)start + rows.y, (int64_t)cap);
    const int blk = start / KV_B + at_block.i;
    const int t0 = blk * KV_B;
    if (t0 >= end || rows.y == 0) return;  // (without rows: its page may be another's by now)
    const int pg = a.table[(int64_t)b * a.cols + a.by_bpp.div(blk)];  // looked at once the input is on its way
    const KvTokens src = tensor ? a.V : a.K;
    const T *x = static_cast<const T *>(src.x) + (int64_t)(rows.x - start + t0) * src.token + (int64_t)h * src.head;
    const int lo = max(start - t0, 0), hi = min(end - t0, KV_B);  // the block's new tokens
    const bool there = pg >= 0 && pg < a.pages;
    uint8_t *rec = a.k + (((int64_t)pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk)) * kv4_bytes(a.d);

    if (tensor == 0) {
        constexpr int NP = D / 32;
        const int g = lane >> 2, c = lane & 3;
        uint32_t raw[NP][2][W];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                // (dims past the last: the first ones once more, which does not change the range)
                const int t = g + 8 * k, dim = 32 * p + 8 * c, from = dim < a.d ? dim : 8 * (c & 1);
#pragma unroll
                for (int i = 0; i < W; ++i) raw[p][k][i] = 0;
                if (t >= lo && t < hi) load8(x + (int64_t)t * src.token + from, src.wide, raw[p][k]);
            }
        if (!there) return;
        Lvq v[2];
        Range r[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            r[k] = range8<T>(raw[0][k]);
#pragma unroll
            for (int p = 1; p < NP; ++p) r[k] = both(r[k], range8<T>(raw[p][k]));
            r[k] = across(across(r[k], 1), 2);
        }
        const bool clip = !__all_sync(0xffffffffu, ordinary(r[0]) && ordinary(r[1]));
        if (clip) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float2 f = make_float2(INFINITY, -INFINITY);
#pragma unroll
                for (int p = 0; p < NP; ++p) f = finite8<T>(raw[p][k], f);
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    f.x = fminf(f.x, __shfl_xor_sync(0xffffffffu, f.x, o));
                    f.y = fmaxf(f.y, __shfl_xor_sync(0xffffffffu, f.y, o));
                }
                r[k] = clipped(f);
            }
        }
        uint32_t fresh = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int t = g + 8 * k;
            v[k] = lvq_of(r[k]);
            if (t < lo || t >= hi) continue;
            fresh |= 0x00ff00ffu << (8 * k);
            if (c == 0) *reinterpret_cast<uint32_t *>(rec + KV_B * a.d + 8 * t) = held(v[k]);
        }
        if (!fresh) return;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (32 * p + 8 * c >= a.d) break;
            float2 n[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (clip) codes8_clipped<T>(raw[p][k], v[k], r[k].lo, r[k].hi, n[k]);
                else codes8<T>(raw[p][k], v[k], n[k]);
            }
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 u = pack2(pack2(n[0][2 * i], n[0][2 * i + 1], 16.0f), pack2(n[1][2 * i], n[1][2 * i + 1], 16.0f), 256.0f);
                w[i] = word_of(u.x, u.y);
            }
            uint2 *dst = reinterpret_cast<uint2 *>(rec + (2 * p + (c >> 1)) * 128 + g * 16 + (c & 1) * 8);
            if (fresh != 0xffffffffu) {
                const uint2 was = *dst;
                w[0] = merged(was.x, w[0], fresh), w[1] = merged(was.y, w[1], fresh);
            }
            *dst = make_uint2(w[0], w[1]);
        }
    } else {
        constexpr int NI = (D + 63) / 64;
        const int c = lane & 3;
        uint32_t raw[NI][4][W];
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1) + 8 * (k >> 1), e = (lane >> 2) + 8 * i, from = 8 * (8 * e < a.d ? e : e & 1);
#pragma unroll
                for (int j = 0; j < W; ++j) raw[i][k][j] = 0;
                if (t >= lo && t < hi) load8(x + (int64_t)t * src.token + from, src.wide, raw[i][k]);
            }
        if (!there) return;
        Range r[4];
        bool fine = true;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            r[k] = range8<T>(raw[0][k]);
#pragma unroll
            for (int i = 1; i < NI; ++i) r[k] = both(r[k], range8<T>(raw[i][k]));
            r[k] = across(across(across(r[k], 4), 8), 16);
            fine = fine && ordinary(r[k]);
        }
        const bool clip = !__all_sync(0xffffffffu, fine);
        if (clip) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float2 f = make_float2(INFINITY, -INFINITY);
#pragma unroll
                for (int i = 0; i < NI; ++i) f = finite8<T>(raw[i][k], f);
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    f.x = fminf(f.x, __shfl_xor_sync(0xffffffffu, f.x, o));
                    f.y = fmaxf(f.y, __shfl_xor_sync(0xffffffffu, f.y, o));
                }
                r[k] = clipped(f);
            }
        }
        Lvq v[4];
        uint32_t fresh = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = 2 * c + (k & 1) + 8 * (k >> 1);
            v[k] = lvq_of(r[k]);
            if (t < lo || t >= hi) continue;
            fresh |= 0x0f0fu << (16 * (k & 1) + 4 * (k >> 1));
            if (lane < 4) *reinterpret_cast<uint32_t *>(rec + KV_B * a.d + 8 * t + 4) = held(v[k]);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int e = (lane >> 2) + 8 * i, odd = e & 1;
            float2 n[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (clip) codes8_clipped<T>(raw[i][k], v[k], r[k].lo, r[k].hi, n[k]);
                else codes8<T>(raw[i][k], v[k], n[k]);
            }
            // dim 8 e + j: bytes 0 and 2 of its word (e even) or 1 and 3
            uint32_t part[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 u = pack2(n[0][j], n[2][j], 16.0f), w = pack2(n[1][j], n[3][j], 16.0f);
                part[2 * j] = word_of(u.x, w.x) << (8 * odd);
                part[2 * j + 1] = word_of(u.y, w.y) << (8 * odd);
            }
            // of the eight words the two lanes share, the even one stores four, the odd one four
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t give = odd ? part[j] : part[j + 4];
                const uint32_t got = __shfl_xor_sync(0xffffffffu, give, 4);
                uint32_t w = (odd ? part[j + 4] : part[j]) | got;
                if (8 * e >= a.d || !fresh) continue;
                uint32_t *dst = reinterpret_cast<uint32_t *>(rec + 8 * a.d + (e >> 1) * 128 + (j + 4 * odd) * 16 + 4 * c);
                if (fresh != 0xffffffffu) w = merged(*dst, w, fresh);
                *dst = w;
            }
        }
    }
}

// the codes in bits 0..3, 16..19 of a word as floats
__device__ __forceinline__ float2 low_codes(uint32_t u) {
    u &= 0x000f000fu;
    return add2(make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442))),
                make_float2(-8388608.0f, -8388608.0f));
}
__device__ __forceinline__ float2 scaled(float2 n, float2 sb) { return fma2(n, make_float2(sb.x, sb.x), make_float2(sb.y, sb.y)); }

// Warps: one a (sequence, block its range reaches, head, tensor).
template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32) kv4_read_kernel(const __grid_constant__ KvCacheArgs a) {
    const int lane = threadIdx.x & 31;
    const int warp = blockIdx.x * WARPS + (threadIdx.x >> 5), tensor = warp & 1;
    T *dst = static_cast<T *>(tensor ? a.outv : a.outk);
    if (!dst) return;
    const int h = a.by_heads.mod(warp >> 1);
    const Place at_block = place_of(a, a.by_heads.div(warp >> 1), lane);
    const int b = at_block.b;
    if (b >= a.batch) return;
    const int2 rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
    const int start = max(a.pos[b], 0);
    const int64_t end = (int64_t)start + rows.y;
    const int blk = start / KV_B + at_block.i;
    const int64_t t0 = (int64_t)blk * KV_B;
    if (t0 >= end) return;
    const int col = a.by_bpp.div(blk);
    const int pg = col < a.cols ? a.table[(int64_t)b * a.cols + col] : -1;
    const bool there = pg >= 0 && pg < a.pages;
    const uint8_t *rec = a.k + (there ? ((int64_t)pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk) : 0) * kv4_bytes(a.d);
    dst += ((rows.x + (t0 - start)) * a.heads + h) * a.d;
    const int64_t step = (int64_t)a.heads * a.d;
    const auto wanted = [&](int t) { return t0 + t >= start && t0 + t < end; };
    const auto scale_of = [&](int t) {  // (scale, bias); an absent page holds zeros
        const uint32_t w = there ? *reinterpret_cast<const uint32_t *>(rec + KV_B * a.d + 8 * t + 4 * tensor) : 0u;
        return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    };

    if (tensor == 0) {
        constexpr int NP = D / 32;
        const int g = lane >> 2, c = lane & 3;
        uint2 w[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            w[p] = make_uint2(0, 0);
            if (there && 32 * p + 8 * c < a.d) w[p] = *reinterpret_cast<const uint2 *>(rec + (2 * p + (c >> 1)) * 128 + g * 16 + (c & 1) * 8);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int t = g + 8 * k;
            if (!wanted(t)) continue;
            const float2 sb = scale_of(t);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                if (32 * p + 8 * c >= a.d) break;
                const uint32_t u = w[p].x >> (8 * k), y = w[p].y >> (8 * k);
                const float2 v[4] = {scaled(low_codes(u), sb), scaled(low_codes(u >> 4), sb), scaled(low_codes(y), sb),
                                     scaled(low_codes(y >> 4), sb)};
                store8(dst + t * step + 32 * p + 8 * c, reinterpret_cast<const float *>(v));
            }
        }
    } else {
        constexpr int NI = (D + 63) / 64;
        const int c = lane & 3;
        uint32_t w[NI][8];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int e = (lane >> 2) + 8 * i;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[i][j] = 0;
                if (there && 8 * e < a.d)
                    w[i][j] = *reinterpret_cast<const uint32_t *>(rec + 8 * a.d + (e >> 1) * 128 + j * 16 + 4 * c) >> (8 * (e & 1));
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {  // tokens 2 c + 8 k and the next
            const int t = 2 * c + 8 * k;
            const bool first = wanted(t), second = wanted(t + 1);
            if (!first && !second) continue;
            const float2 sb0 = scale_of(t), sb1 = scale_of(t + 1);
            const float2 s = make_float2(sb0.x, sb1.x), o = make_float2(sb0.y, sb1.y);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int e = (lane >> 2) + 8 * i;
                if (8 * e >= a.d) break;
                float v0[8], v1[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 y = fma2(low_codes(w[i][j] >> (4 * k)), s, o);
                    v0[j] = y.x, v1[j] = y.y;
                }
                if (first) store8(dst + t * step + 8 * e, v0);
                if (second) store8(dst + (t + 1) * step + 8 * e, v1);
            }
        }
    }
}

}  // namespace

cudaError_t launch_kv4_write(const KvCacheArgs &args, int dtype, cudaStream_t st) {
    const KvCacheArgs a = with_divisions(args);
    const unsigned grid = (unsigned)grid_of(a);
    if (a.d <= 64) KV_BY_TYPE(kv4_write_kernel, 64);
    else if (a.d <= 128) KV_BY_TYPE(kv4_write_kernel, 128);
    else KV_BY_TYPE(kv4_write_kernel, 256);
    return launched();
}

cudaError_t launch_kv4_read(const KvCacheArgs &args, int dtype, cudaStream_t st) {
    const KvCacheArgs a = with_divisions(args);
    const unsigned grid = (unsigned)grid_of(a);
    if (a.d <= 64) KV_BY_TYPE(kv4_read_kernel, 64);
    else if (a.d <= 128) KV_BY_TYPE(kv4_read_kernel, 128);
    else KV_BY_TYPE(kv4_read_kernel, 256);
    return launched();
}

}  // namespace skm
