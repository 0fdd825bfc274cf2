// Writing keys and values into the 4-bit cache and reading them back.
//
// A token's key (or value) of a head is one LVQ vector: bias b, the largest f16 not above its
// smallest element, scale s, the smallest f16 with b + 15 s not below its largest, codes
// rint((x - b) / s).  One warp takes one block (16 tokens) of one head's keys or values: a first pass for smallest and
// largest, in registers and over a few lanes, a second one, out of L1, for the codes (HBM is read once).
// A vector's codes depend on nothing else: what the block holds is never rounded again.
//
// Lanes.  Ranges, and keys' codes: (g, c), tokens g and g + 8, of every 32 dims the eight from 8 c on: a token's 32 dims
// are 64 consecutive bytes of 16-bit input, and the lane's codes are two neighbouring words.
// Values: (e, c), dims 8 e .. of the four tokens 2c, 2c + 1, 2c + 8, 2c + 9 that share a word; the
// other dims of a word are those of the lane next to it in e.
//
// Rounding.  q = d y, d = x - b and y the correctly rounded reciprocal of s: three roundings, so q, 15 at most, is within
// 45 2^-24 of the quotient and its nearest integer is the quotient's unless it lies within 2^-18 of the middle of two.  It
// often is the middle itself (16-bit values, biases and scales have few bits: one value in 2500 of a bf16 input): then q
// corrected by its remainder, q + (d - q s) y, is k + 1/2, the remainder of that is 0, d is exact, and half to even is
// right; else x - b is compared with (k + 1/2) s in 64 bits, and where the two are equal what x - b was rounded by decides.
// 2^23 + q is an integer, rounded half to even; codes become words by multiply-adds of integers as floats (below 2^16
// beside 2^23, exact), two at a time.
//
// What bounds them.  Writing: instructions (a value's code takes 10 in packed pairs, its place in a word 2 more; issue
// slots 55% taken) and reads that not enough warps wait for; 12 prompts of up to 2500 tokens, 8 heads of 128 dims, bf16: 42
// us and 2.6 TB/s of the kernel, 65 us with reading back.  Quotients as divisions, or corrected everywhere, and zeros for rows
// that are not new took 71; two, four and eight heads a warp with the next one's rows prefetched 69, 72 and 78 (their
// loop's registers are too many).  Reading: HBM; 4 sequences of up to 32768 tokens, 82 us, 93% of a copy's rate.
#include "skm_kv_cache.cuh"

namespace skm {

namespace {

constexpr float MAGIC = 8388608.0f;  // 2^23: x + this, for x from 0 to 2^22, is rint(x) + this
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

// the code of a value within its vector's range, by an exact comparison where fp32 leaves it open
__device__ __forceinline__ float code_of(float x, const Lvq &v) {
    const float q = (x - v.b) * v.inv, c = rintf(q);
    if (fabsf(q - c) <= NEAR) return c;
    const float k = floorf(q);  // near k + 1/2
    const double over = (double)x - (double)v.b, mid = ((double)k + 0.5) * (double)v.s;
    if (over != mid) return over > mid ? k + 1.0f : k;
    // what the difference was rounded by (Knuth's exact sum): x next to 0 and b are further apart than 53 bits
    const double z = __dadd_rn(over, -(double)x), rest = __dadd_rn(__dadd_rn((double)x, -__dadd_rn(over, -z)), __dadd_rn(-(double)v.b, -z));
    return rest > 0.0 || (rest == 0.0 && ((int)k & 1)) ? k + 1.0f : k;
}
// the same of 8 values, in a nibble each (by value and not inlined: what is rare costs the ordinary path no registers)
template <typename T>
struct Eight {
    uint32_t w[WORDS8<T>];
};
template <typename T>
__device__ __noinline__ uint32_t codes8_near(Eight<T> x, float b, float s, float inv) {
    const Lvq v{b, s, inv};
    uint32_t c = 0;
    for (int i = 0; i < 4; ++i) {
        const float2 p = value2<T>(x.w, i);
        c |= (uint32_t)code_of(p.x, v) << (8 * i) | (uint32_t)code_of(p.y, v) << (8 * i + 4);
    }
    return c;
}
// x - b without a rounding error (Knuth's exact sum)
__device__ __forceinline__ bool exact_less(float x, float b, float d) {
    const float z = __fadd_rn(d, -x);
    return __fadd_rn(__fadd_rn(x, -__fadd_rn(d, -z)), __fadd_rn(-b, -z)) == 0.0f;
}
// codes of 8 values as floats, pairs i with bit i of UP + 2^23
template <int UP, typename T>
__device__ __forceinline__ void codes8(const Eight<T> &x, const Lvq &v, float2 (&c)[4]) {
    const float2 less = make_float2(-v.b, -v.b), by = make_float2(v.inv, v.inv);
    const float2 up = make_float2(MAGIC, MAGIC), down = make_float2(-MAGIC, -MAGIC);
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 q = mul2(add2(value2<T>(x.w, i), less), by), t = add2(q, up), n = add2(t, down);
        const float2 off = fma2(n, make_float2(-1.0f, -1.0f), q);
        far = fmaxf(far, fmaxf(fabsf(off.x), fabsf(off.y)));
        c[i] = UP >> i & 1 ? t : n;
    }
    if (far <= NEAR) return;
    // every value once more, from the corrected quotient: a middle counts where it is one exactly
    const float2 s = make_float2(-v.s, -v.s);
    bool open = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = value2<T>(x.w, i), d = add2(y, less), q0 = mul2(d, by), q = fma2(fma2(q0, s, d), by, q0), r = fma2(q, s, d);
        const float2 t = add2(q, up), n = add2(t, down);
        const float ex = fabsf(q.x - n.x), ey = fabsf(q.y - n.y);
        open = open || (ex > NEAR && !(ex == 0.5f && r.x == 0.0f && exact_less(y.x, v.b, d.x)));
        open = open || (ey > NEAR && !(ey == 0.5f && r.y == 0.0f && exact_less(y.y, v.b, d.y)));
        c[i] = UP >> i & 1 ? t : n;
    }
    if (open) {
        const uint32_t n = codes8_near<T>(x, v.b, v.s, v.inv);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float more = UP >> i & 1 ? MAGIC : 0.0f;
            c[i] = make_float2((float)(n >> (8 * i) & 15) + more, (float)(n >> (8 * i + 4) & 15) + more);
        }
    }
}

__device__ __forceinline__ float2 pack2(float2 a, float2 b, float up) { return fma2(b, make_float2(up, up), a); }
// two integers below 2^16, each + 2^23, as the halves of a word
__device__ __forceinline__ uint32_t word_of(float lo, float hi) {
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
}
__device__ __forceinline__ uint32_t merged(uint32_t was, uint32_t now, uint32_t mask) { return (was & ~mask) | (now & mask); }

// A block's new tokens one after the other, whatever they hold, by the definition: for blocks with infinities, NaN,
// values beyond f16 (left out, or clipped, of a vector's range and taken into it: NaN to its smallest), and for
// rows that no wide load may read.
template <typename T>
__device__ __noinline__ void block_slowly(const T *x, int64_t step, int d, int tensor, int lo, int hi, uint8_t *rec, int lane) {
    for (int t = lo; t < hi; ++t) {
        const T *row = x + t * step;
        const auto at = [&](int dim) {
            if constexpr (std::is_same<T, float>::value) return row[dim];
            else if constexpr (std::is_same<T, __half>::value) return __half2float(row[dim]);
            else return __bfloat162float(row[dim]);
        };
        float least = INFINITY, most = -INFINITY;
        for (int i = lane; i < d; i += 32) {
            const float y = at(i);
            if (fabsf(y) < INFINITY) least = fminf(least, y), most = fmaxf(most, y);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        }
        Range r{0.0f, 0.0f};  // without a finite element
        if (least <= most) r = Range{fminf(fmaxf(least, -F16_MOST), F16_MOST), fminf(fmaxf(most, -F16_MOST), F16_MOST)};
        const Lvq v = lvq_of(r);
        const auto code = [&](int dim) -> uint32_t {
            float y = at(dim);
            y = y == y ? fminf(fmaxf(y, r.lo), r.hi) : r.lo;
            return (uint32_t)code_of(y, v);
        };
        if (tensor == 0) {
            for (int i = lane; i < d / 2; i += 32) {  // a byte: two dims of the token
                const int w = i >> 3, c = (i >> 1) & 3, l = i & 1, dim = 16 * w + 4 * c + l;
                rec[128 * w + 16 * (t & 7) + 4 * c + 2 * l + (t >> 3)] = (uint8_t)(code(dim) | code(dim + 2) << 4);
            }
        } else {
            for (int dim = lane; dim < d; dim += 32) {  // half a byte
                uint8_t *p = rec + 8 * d + 128 * (dim >> 4) + 16 * (dim & 7) + 4 * ((t & 7) >> 1) + 2 * (t & 1) + ((dim >> 3) & 1);
                const int up = 4 * (t >> 3);
                *p = (uint8_t)((*p & ~(15u << up)) | code(dim) << up);
            }
        }
        if (lane == 0) *reinterpret_cast<uint32_t *>(rec + KV_B * d + 8 * t + 4 * tensor) = held(v);
    }
}

// Warps: one a (sequence, block its new rows reach, head, tensor).  D: dims at most
template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32, sizeof(T) * D <= 256 ? 12 : sizeof(T) * D <= 512 ? 8 : 4)
    kv4_write_kernel(const __grid_constant__ KvCacheArgs a) {
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
    uint8_t *rec = a.k + (((int64_t)(there ? pg : 0) * a.heads + h) * a.bpp + a.by_bpp.mod(blk)) * kv4_bytes(a.d);
    // 8 values of a token (if it is not new, of the new one next to it, whose codes are not stored for it); where wide
    // loads are not possible all blocks go the slow way
    const auto row_of = [&](int t) { return x + (int64_t)min(max(t, lo), hi - 1) * src.token; };
    const auto get = [&](const T *row, int dim) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + dim);
        Eight<T> e;
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const uint4 y = __ldg(p + i / 4);
            e.w[i] = y.x, e.w[i + 1] = y.y, e.w[i + 2] = y.z, e.w[i + 3] = y.w;
        }
        return e;
    };
    if (!src.wide) {
        if (there) block_slowly(x, src.token, a.d, tensor, lo, hi, rec, lane);
        return;
    }
    // the range of each token, in lanes (g, c) of either tensor: tokens g and g + 8, of every 32 dims the eight from 8 c on
    const int g = lane >> 2, c = lane & 3;
    constexpr int NP = D / 32;
    Range r[2];
    const T *const row[2] = {row_of(g), row_of(g + 8)};
    {
        Eight<T> raw[NP][2];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                // (dims past the last: the first ones once more, which does not change the range)
                const int dim = 32 * p + 8 * c;
                raw[p][k] = get(row[k], dim < a.d ? dim : 8 * (c & 1));
            }
        if (!there) return;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            r[k] = range8<T>(raw[0][k].w);
#pragma unroll
            for (int p = 1; p < NP; ++p) r[k] = both(r[k], range8<T>(raw[p][k].w));
            r[k] = across(across(r[k], 1), 2);
        }
    }
    if (!__all_sync(0xffffffffu, ordinary(r[0]) && ordinary(r[1]))) {
        block_slowly(x, src.token, a.d, tensor, lo, hi, rec, lane);
        return;
    }
    Lvq v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int t = g + 8 * k;
        v[k] = lvq_of(r[k]);
        if (c == 0 && t >= lo && t < hi) *reinterpret_cast<uint32_t *>(rec + KV_B * a.d + 8 * t + 4 * tensor) = held(v[k]);
    }
    // the codes: the values again, out of L1, in rolled loops (unrolled, with the values in registers, warps waited for
    // their instructions most of all: writing and reading back 87 us)
    if (tensor == 0) {
        uint32_t fresh = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) fresh |= g + 8 * k >= lo && g + 8 * k < hi ? 0x00ff00ffu << (8 * k) : 0u;
        if (!fresh) return;
#pragma unroll 1
        for (int dim = 8 * c; dim < a.d; dim += 32) {
            float2 n[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (k) codes8<0>(get(row[k], dim), v[k], n[k]);
                else codes8<5>(get(row[k], dim), v[k], n[k]);
            }
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 u = pack2(pack2(n[0][2 * i], n[0][2 * i + 1], 16.0f), pack2(n[1][2 * i], n[1][2 * i + 1], 16.0f), 256.0f);
                w[i] = word_of(u.x, u.y);
            }
            uint2 *dst = reinterpret_cast<uint2 *>(rec + (dim >> 4) * 128 + g * 16 + (c & 1) * 8);
            if (fresh != 0xffffffffu) {
                const uint2 was = *dst;
                w[0] = merged(was.x, w[0], fresh), w[1] = merged(was.y, w[1], fresh);
            }
            *dst = make_uint2(w[0], w[1]);
        }
    } else {
        // lanes (e, c): dims 8 e .. of the four tokens that share a word; their vectors from the lanes above
        Lvq u[4];
        uint32_t fresh = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = 2 * c + (k & 1) + 8 * (k >> 1), from = 4 * (2 * c + (k & 1));
            u[k].b = __shfl_sync(0xffffffffu, v[k >> 1].b, from);
            u[k].s = __shfl_sync(0xffffffffu, v[k >> 1].s, from);
            u[k].inv = __shfl_sync(0xffffffffu, v[k >> 1].inv, from);
            fresh |= t >= lo && t < hi ? 0x0f0fu << (16 * (k & 1) + 4 * (k >> 1)) : 0u;
        }
        const int odd = g & 1;
        const T *const from[4] = {row_of(2 * c), row_of(2 * c + 1), row_of(2 * c + 8), row_of(2 * c + 9)};
#pragma unroll 1
        for (int e0 = 0; 8 * e0 < a.d; e0 += 8) {
            const int e = e0 + g;
            const bool in = 8 * e < a.d && fresh;
            // dim 8 e + j: bytes 0 and 2 of its word (e even) or 1 and 3
            float2 n[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float2 first[4], second[4];
                codes8<15>(get(from[k], in ? 8 * e : 0), u[k], first);
                codes8<0>(get(from[k + 2], in ? 8 * e : 0), u[k + 2], second);
#pragma unroll
                for (int j = 0; j < 4; ++j) n[k][j] = pack2(first[j], second[j], 16.0f);
            }
            uint32_t part[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                part[2 * j] = word_of(n[0][j].x, n[1][j].x) << (8 * odd);
                part[2 * j + 1] = word_of(n[0][j].y, n[1][j].y) << (8 * odd);
            }
            // of the eight words the two lanes share, the even one stores four, the odd one four
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t give = odd ? part[j] : part[j + 4];
                const uint32_t got = __shfl_xor_sync(0xffffffffu, give, 4);
                uint32_t w = (odd ? part[j + 4] : part[j]) | got;
                if (!in) continue;
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
// 8 values; f16's end at its largest number (which a vector's largest code may stand for more than: -65504 to 65504 gives 65536)
template <typename T>
__device__ __forceinline__ void store8_within(T *p, const float *v) {
    if constexpr (std::is_same<T, __half>::value) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = kv_f16_within(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        store8(p, v);
    }
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
                store8_within(dst + t * step + 32 * p + 8 * c, reinterpret_cast<const float *>(v));
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
                if (first) store8_within(dst + t * step + 8 * e, v0);
                if (second) store8_within(dst + (t + 1) * step + 8 * e, v1);
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
