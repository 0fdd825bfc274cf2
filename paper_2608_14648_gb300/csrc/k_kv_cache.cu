// Writing keys and values into the 8-bit cache and reading them back.
//
// One warp takes one block (16 tokens) of one head's keys or values: a first pass over
// the block's new values for the largest magnitude, a second one, out of L1, for the
// codes.  A warp needs no other warp, so an append (one token, a warp busy for its memory
// latencies) and a prompt (thousands of independent 4 KB reads in flight) are the
// same code.  What bounds writing is how many of those reads are in flight and the
// instructions of a block (1095 a warp for 2048 values): the input is read before the page is known, eight
// 16-byte loads a lane at a time, and the second pass is a rolled loop (holding the
// values in registers instead took an unrolled path for each d, and warps waited for
// its instructions: 43 us against 37 for the 12 prompts below).  64 registers, 32 warps an
// SM: with 48 or 40 registers the loads in flight cost more than the warps give (writing and reading
// back 54, 55 and 59 us).
//
// Measured (GB300, bf16, 8 heads of 128): writing 12 prompts of up to 2500 tokens, 93 MB
// in and out, 32 us = 2.9 TB/s; reading 4 sequences of up to 32768 tokens back, 611 MB,
// 101 us = 6.0 TB/s (a plain copy: 6.8).
//
// Lanes: the magnitudes and the keys along d (a 16-byte code store, two 16-byte loads
// of 16-bit values); values, whose blocks keep the 16 tokens of a dim together, 8
// dims of the four tokens that share a 32-bit word, so the transposition stays in
// registers.
//
// The largest magnitude is an integer maximum of the values' bits without
// their sign, in which infinities and NaN come out on top: a warp that finds one
// goes element by element.
//
// Rounding: code = rint(x / scale) with the quotient rounded to fp32.  The quotient is
// q = x y, y the correctly rounded reciprocal, corrected twice by its exact
// remainder: q' = q + (x - q s) y.  q is within 1.5 units in the last place, the first correction
// within one, and by Markstein's theorem (IBM J. Res. Dev. 34, 1990) the second
// is the quotient as a division rounds it.  Five operations, two values at a time; a
// division only where x y lies near the middle of two codes took longer (37 us
// against 32), because 16-bit values meet it often (half the largest one is 63.5).
#include <algorithm>
#include <type_traits>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int WARPS = 8;
constexpr float CODE_MAGIC = 12583040.0f;  // 1.5 2^23 + 128: q + this holds rint(q) + 128 in its low byte

template <typename T>
constexpr int WORDS8 = 8 * sizeof(T) / 4;  // words of 8 values
template <typename T>
constexpr uint32_t INF_BITS = std::is_same<T, float>::value ? 0x7f800000u : std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;

// 16 bytes without the alignment of a vector (not inlined: the loads would be
// predicated into the aligned path)
template <typename T>
__device__ __noinline__ uint4 load_slowly(const T *p) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
        for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
    } else {
        const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
        for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 8 consecutive values as they are
template <typename T>
__device__ __forceinline__ void load8(const T *p, int wide, uint32_t *w) {
#pragma unroll
    for (int i = 0; i < WORDS8<T>; i += 4) {
        const T *q = p + i * (4 / (int)sizeof(T));
        const uint4 a = wide ? *reinterpret_cast<const uint4 *>(q) : load_slowly(q);
        w[i] = a.x, w[i + 1] = a.y, w[i + 2] = a.z, w[i + 3] = a.w;
    }
}
// value i of words
template <typename T>
__device__ __forceinline__ float value(const uint32_t *w, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    const uint32_t x = w[i >> 1];
    if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((uint16_t)(i & 1 ? x >> 16 : x)));
    return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
}
// the larger magnitudes' bits, a 16-bit pair at a time
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t m, uint32_t w) {
    if constexpr (sizeof(T) == 4) return max(m, w & 0x7fffffffu);
    return __vmaxu2(m, w & 0x7fff7fffu);
}
template <typename T>
__device__ __forceinline__ float magnitude(uint32_t bits) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
    if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((uint16_t)bits));
    return __uint_as_float(bits << 16);
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const float *v) {
    if constexpr (std::is_same<T, float>::value) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __noinline__ uint32_t code_exact(float x, float s) {
    float q = __fdiv_rn(x, s);
    q = q == q ? fminf(fmaxf(rintf(q), -127.0f), 127.0f) : 0.0f;
    return (uint32_t)(int)(q + 128.0f);
}

// codes of four values in a word, the first in the low byte; quick: they are
// finite, and s and its reciprocal far from the ends of the exponent's range
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float s, float inv, bool quick) {
    if (!quick) {
        if (!(s > 0.0f)) return 0x80808080u;
        return code_exact(a, s) | code_exact(b, s) << 8 | code_exact(c, s) << 16 | code_exact(d, s) << 24;
    }
    const float2 y = make_float2(inv, inv), less = make_float2(-s, -s);
    const auto codes2 = [&](float2 x) {
        float2 q = mul2(x, y);
        q = fma2(fma2(q, less, x), y, q);
        q = fma2(fma2(q, less, x), y, q);
        q = add2(q, make_float2(CODE_MAGIC, CODE_MAGIC));
        return __byte_perm(__float_as_uint(q.x), __float_as_uint(q.y), 0x0040);
    };
    return __byte_perm(codes2(make_float2(a, b)), codes2(make_float2(c, d)), 0x5410);
}

// codes of a word of the block's earlier tokens after its scale grew by 1 / r
__device__ __forceinline__ uint32_t rescale4(uint32_t word, float r) {
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) out |= (uint32_t)(int)(rintf(kv_code(word, i) * r) + 128.0f) << (8 * i);
    return out;
}

// The block's scale: bits = the lane's largest magnitudes, finite(): its
// largest finite one (rare)
struct BlockScale {
    float s, inv, ratio;  // ratio: old / s, 1 when the codes held stay as they are
    bool quick;
};
template <typename T, typename Finite>
__device__ __forceinline__ BlockScale block_scale(uint32_t bits, float old, Finite finite) {
    if constexpr (sizeof(T) == 2) bits = max(bits & 0xffffu, bits >> 16);
    bits = __reduce_max_sync(0xffffffffu, bits);
    BlockScale b;
    b.quick = bits < INF_BITS<T>;
    float a = magnitude<T>(bits);
    if (!b.quick) a = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(finite())));
    b.s = fmaxf(old, a * (1.0f / 127.0f));
    b.ratio = old > 0.0f && b.s > old ? __fdiv_rn(old, b.s) : 1.0f;
    b.quick = b.quick && b.s > 1e-30f;  // (smaller: a remainder may be subnormal)
    b.inv = b.quick ? __frcp_rn(b.s) : 0.0f;
    return b;
}

// Which block a warp takes: its sequence and how many blocks after the first.
// Up to 32 sequences, the blocks there are, in order; more, a row of
// most_blocks for each.
struct Place {
    int b, i;
};
__device__ __forceinline__ Place place_of(const KvCacheArgs &a, int u, int lane) {
    if (a.batch > 32) return Place{a.by_most.div(u), a.by_most.mod(u)};
    int n = 0;
    if (lane < a.batch) {
        const int2 rows = kv_rows_of(a.cu, lane, a.tokens, a.max_tokens);
        const int start = max(a.pos[lane], 0);
        if (rows.y > 0) n = (start % KV_B + rows.y + KV_B - 1) / KV_B;
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    const uint32_t after = __ballot_sync(0xffffffffu, x > u);  // the first whose blocks reach past u
    const int b = after ? __ffs(after) - 1 : a.batch;
    return Place{b, u - __shfl_sync(0xffffffffu, x - n, b & 31)};
}

// Warps: one a (sequence, block its new rows reach, head, tensor).
template <typename T>
__global__ void __launch_bounds__(WARPS * 32, 4) kv_write_kernel(const __grid_constant__ KvCacheArgs a) {
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

    // the largest magnitude: 8 values a lane, consecutive lanes along d
    uint32_t top = 0;
    const int eighths = KV_B * (a.d / 8);
    constexpr int W = WORDS8<T>;
    const auto loads = [&](auto many, bool wide) {
        constexpr int AT_ONCE = decltype(many)::value;
#pragma unroll 1
        for (int q0 = lane; q0 < eighths; q0 += 32 * AT_ONCE) {
            uint32_t v[AT_ONCE][W];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int q = q0 + 32 * i, t = a.by_eighths.div(q);
#pragma unroll
                for (int j = 0; j < W; ++j) v[i][j] = 0;
                if (t >= lo && t < hi) load8(x + (int64_t)t * src.token + 8 * (q - t * (a.d / 8)), wide, v[i]);
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) top = larger<T>(top, v[i][j]);
        }
    };
    if (src.wide) loads(std::integral_constant<int, 32 / W>{}, true);
    else loads(std::integral_constant<int, 1>{}, false);
    if (pg < 0 || pg >= a.pages) return;
    const int64_t at = ((int64_t)pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk);
    uint8_t *codes = (tensor ? a.v : a.k) + at * (KV_B * a.d);
    float *where = reinterpret_cast<float *>(a.scales + at) + tensor;
    const float old = lo > 0 ? *where : 0.0f;
    const BlockScale bs = block_scale<T>(top, old, [&] {
        float m = 0.0f;
        for (int q = lane; q < eighths; q += 32) {
            const int t = a.by_eighths.div(q);
            if (t < lo || t >= hi) continue;
            uint32_t v[W];
            load8(x + (int64_t)t * src.token + 8 * (q - t * (a.d / 8)), src.wide, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = fabsf(value<T>(v, j));
                m = y < INFINITY ? fmaxf(m, y) : m;
            }
        }
        return m;
    });
    __syncwarp();
    if (lane == 0) *where = bs.s;

    // the codes: the values again, out of L1
    if (tensor == 0) {
        const int nc = a.d / KV_B;
#pragma unroll 1
        for (int q = lane; q < KV_B * nc; q += 32) {
            const int t = a.by_chunks.div(q), w = q - t * nc;
            uint4 *p = reinterpret_cast<uint4 *>(codes + w * 256 + t * 16);
            if (t >= lo && t < hi) {
                uint32_t v[2 * W], c[4];
                load8(x + (int64_t)t * src.token + 16 * w, src.wide, v);
                load8(x + (int64_t)t * src.token + 16 * w + 8, src.wide, v + W);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    c[j] = codes4(value<T>(v, 4 * j), value<T>(v, 4 * j + 1), value<T>(v, 4 * j + 2),
                                  value<T>(v, 4 * j + 3), bs.s, bs.inv, bs.quick);
                *p = make_uint4(c[0], c[1], c[2], c[3]);
            } else if (t < lo && bs.ratio != 1.0f) {
                const uint4 c = *p;
                *p = make_uint4(rescale4(c.x, bs.ratio), rescale4(c.y, bs.ratio), rescale4(c.z, bs.ratio),
                                rescale4(c.w, bs.ratio));
            }
        }
    } else {
#pragma unroll 1
        for (int q = lane; q < a.d / 2; q += 32) {
            const int c = q & 3, e = q >> 2;
            uint32_t v[4][W];
            uint32_t fresh = 0, held = 0;  // bytes of new tokens, of tokens from before
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1) + 8 * (k >> 1);
#pragma unroll
                for (int j = 0; j < W; ++j) v[k][j] = 0;
                if (t >= lo && t < hi) {
                    load8(x + (int64_t)t * src.token + 8 * e, src.wide, v[k]);
                    fresh |= 0xffu << (8 * k);
                }
                if (t < lo) held |= 0xffu << (8 * k);
            }
            if (!fresh && (!held || bs.ratio == 1.0f)) continue;
            uint32_t *p = reinterpret_cast<uint32_t *>(codes + 8 * e * 16 + 4 * c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t w = codes4(value<T>(v[0], j), value<T>(v[1], j), value<T>(v[2], j), value<T>(v[3], j),
                                    bs.s, bs.inv, bs.quick);
                if (fresh != 0xffffffffu) {
                    const uint32_t was = p[4 * j];
                    const uint32_t kept = bs.ratio != 1.0f ? rescale4(was, bs.ratio) : was;
                    w = (w & fresh) | (kept & held) | (was & ~(fresh | held));
                }
                p[4 * j] = w;
            }
        }
    }
}

// Warps: one a (sequence, block its range reaches, head, tensor).
template <typename T, int NU>
__global__ void __launch_bounds__(WARPS * 32) kv_read_kernel(const __grid_constant__ KvCacheArgs a) {
    T *dst = static_cast<T *>(blockIdx.x * WARPS + (threadIdx.x >> 5) & 1 ? a.outv : a.outk);
    if (!dst) return;
    const int lane = threadIdx.x & 31;
    const int warp = blockIdx.x * WARPS + (threadIdx.x >> 5), tensor = warp & 1;
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
    const int64_t at = there ? ((int64_t)pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk) : 0;
    const int nc = a.d / KV_B;
    const uint8_t *codes = (tensor ? a.v : a.k) + at * (KV_B * a.d);
    const float s = there ? reinterpret_cast<const float *>(a.scales + at)[tensor] : 0.0f;
    dst += ((rows.x + (t0 - start)) * a.heads + h) * a.d;
    const int64_t step = (int64_t)a.heads * a.d;
    const auto wanted = [&](int t) { return t0 + t >= start && t0 + t < end; };

    if (tensor == 0) {
        uint4 c[NU];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = a.by_chunks.div(q), w = q - t * nc;
            c[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
            if (there && t < KV_B && wanted(t)) c[i] = *reinterpret_cast<const uint4 *>(codes + w * 256 + t * 16);
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = a.by_chunks.div(q), w = q - t * nc;
            if (t >= KV_B || !wanted(t)) continue;
            const uint32_t word[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = s * kv_code(word[j >> 2], j & 3);
            store8(dst + t * step + 16 * w, v);
            store8(dst + t * step + 16 * w + 8, v + 8);
        }
    } else {
        constexpr int NV = (NU + 1) / 2;
        const int last = a.d / 2;
        uint32_t c[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = lane + 32 * i, k = q & 3, e = q >> 2;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                c[i][j] = 0x80808080u;
                if (there && q < last) c[i][j] = *reinterpret_cast<const uint32_t *>(codes + (8 * e + j) * 16 + 4 * k);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = lane + 32 * i, k = q & 3, e = q >> 2;
            if (q >= last) continue;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int t = 2 * k + (m & 1) + 8 * (m >> 1);
                if (!wanted(t)) continue;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = s * kv_code(c[i][j], m);
                store8(dst + t * step + 8 * e, v);
            }
        }
    }
}

// blocks that max_tokens rows reach at most, wherever the first one lies
int most_blocks_of(const KvCacheArgs &a) { return (int)(((int64_t)a.max_tokens + KV_B - 1 + KV_B - 1) / KV_B); }

// at most: the blocks of a row for each sequence, and those that the tokens fill and touch
int64_t grid_of(const KvCacheArgs &a) {
    int64_t blocks = (int64_t)a.batch * most_blocks_of(a);
    if (a.batch <= 32) blocks = std::min<int64_t>(blocks, a.tokens / KV_B + 2 * (int64_t)a.batch);
    return cdiv(blocks * a.heads * 2, WARPS);
}

}  // namespace

#define KV_BY_TYPE(KERNEL, ...)                                                                             \
    do {                                                                                                    \
        if (dtype == SKM_DTYPE_F32) KERNEL<float __VA_OPT__(, ) __VA_ARGS__><<<grid, WARPS * 32, 0, st>>>(a); \
        else if (dtype == SKM_DTYPE_BF16)                                                                   \
            KERNEL<__nv_bfloat16 __VA_OPT__(, ) __VA_ARGS__><<<grid, WARPS * 32, 0, st>>>(a);               \
        else KERNEL<__half __VA_OPT__(, ) __VA_ARGS__><<<grid, WARPS * 32, 0, st>>>(a);                     \
    } while (0)

static KvCacheArgs with_divisions(KvCacheArgs a) {
    a.by_heads = FastDiv(a.heads);
    a.by_bpp = FastDiv(a.bpp);
    a.by_most = FastDiv(most_blocks_of(a));
    a.by_chunks = FastDiv(a.d / KV_B);
    a.by_eighths = FastDiv(a.d / 8);
    return a;
}

cudaError_t launch_kv_write(const KvCacheArgs &args, int dtype, cudaStream_t st) {
    const KvCacheArgs a = with_divisions(args);
    const unsigned grid = (unsigned)grid_of(a);
    KV_BY_TYPE(kv_write_kernel);
    return launched();
}

cudaError_t launch_kv_read(const KvCacheArgs &args, int dtype, cudaStream_t st) {
    const KvCacheArgs a = with_divisions(args);
    const unsigned grid = (unsigned)grid_of(a);
    if (a.d <= 64) KV_BY_TYPE(kv_read_kernel, 2);
    else if (a.d <= 128) KV_BY_TYPE(kv_read_kernel, 4);
    else KV_BY_TYPE(kv_read_kernel, 8);
    return launched();
}

}  // namespace skm
