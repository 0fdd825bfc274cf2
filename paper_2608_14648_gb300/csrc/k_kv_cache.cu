// Writing keys and values into the 8-bit cache and reading them back.
//
// One warp takes one block (16 tokens) of one head's keys or values: it holds
// the block's new values in registers as they came, so the largest magnitude,
// the scale and the codes come from one read of the input.  Both kernels move
// bytes; a warp needs no other warp, so an append (one token, a warp busy for its
// memory latencies) and a prompt (thousands of independent 4 KB reads in flight) are
// the same code.  What bounds writing is how many of those reads are in flight:
// the input is read before the page is known, and 16-bit values stay packed
// (64 registers, 32 warps an SM).
//
// Lanes: keys, a unit is 16 dims of a token (a 16-byte code store, two 16-byte
// loads of 16-bit values), consecutive lanes along d; values, whose blocks
// keep the 16 tokens of a dim together, a unit is 8 dims of the four tokens
// that share a 32-bit word, so the transposition stays in registers.
//
// The largest magnitude is an integer maximum of the values' bits without
// their sign, in which infinities and NaN come out on top: a warp that finds one
// goes element by element.
//
// Rounding: code = rint(x / scale) with the quotient rounded to fp32.  x times
// the reciprocal is within 1.6e-5 of x / scale (|quotient| < 128, two roundings
// of 2^-24 relative), the fp32 quotient within 8e-6, so both round to the same
// integer unless x times the reciprocal lies within 3e-5 of a half; only those
// elements take the division.
#include <algorithm>
#include <type_traits>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int WARPS = 8;
constexpr float CODE_MAGIC = 12583040.0f;  // 1.5 2^23 + 128: q + this holds rint(q) + 128 in its low byte
constexpr float NEAR_HALF = 0.49997f;

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
// finite and the reciprocal of s is a normal number
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float s, float inv, bool quick) {
    if (!quick) {
        if (!(s > 0.0f)) return 0x80808080u;
        return code_exact(a, s) | code_exact(b, s) << 8 | code_exact(c, s) << 16 | code_exact(d, s) << 24;
    }
    const float fa = fmaf(a, inv, CODE_MAGIC), fb = fmaf(b, inv, CODE_MAGIC);
    const float fc = fmaf(c, inv, CODE_MAGIC), fd = fmaf(d, inv, CODE_MAGIC);
    const float ra = fmaf(a, inv, CODE_MAGIC - fa), rb = fmaf(b, inv, CODE_MAGIC - fb);
    const float rc = fmaf(c, inv, CODE_MAGIC - fc), rd = fmaf(d, inv, CODE_MAGIC - fd);
    const uint32_t lo = __byte_perm(__float_as_uint(fa), __float_as_uint(fb), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(fc), __float_as_uint(fd), 0x0040);
    uint32_t w = __byte_perm(lo, hi, 0x5410);
    if (fmaxf(fmaxf(fabsf(ra), fabsf(rb)), fmaxf(fabsf(rc), fabsf(rd))) > NEAR_HALF) {
        if (fabsf(ra) > NEAR_HALF) w = (w & 0xffffff00u) | code_exact(a, s);
        if (fabsf(rb) > NEAR_HALF) w = (w & 0xffff00ffu) | code_exact(b, s) << 8;
        if (fabsf(rc) > NEAR_HALF) w = (w & 0xff00ffffu) | code_exact(c, s) << 16;
        if (fabsf(rd) > NEAR_HALF) w = (w & 0x00ffffffu) | code_exact(d, s) << 24;
    }
    return w;
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
    b.quick = b.quick && b.s > 1e-37f;
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

// Warps: one a (sequence, block its new rows reach, head, tensor).  NU: units a lane.
template <typename T, int NU>
__global__ void __launch_bounds__(WARPS * 32) kv_write_kernel(const __grid_constant__ KvCacheArgs a) {
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
    const int nc = a.d / KV_B;
    const KvTokens src = tensor ? a.V : a.K;
    const T *x = static_cast<const T *>(src.x) + (int64_t)(rows.x - start + t0) * src.token + (int64_t)h * src.head;
    const bool holds = start > t0;
    const bool full = !holds && t0 + KV_B <= end;
    uint32_t top = 0;
    uint8_t *codes = nullptr;
    float *where = nullptr;
    const auto find = [&] {  // false: an absent page
        if (pg < 0 || pg >= a.pages) return false;
        const int64_t at = ((int64_t)pg * a.heads + h) * a.bpp + a.by_bpp.mod(blk);
        codes = (tensor ? a.v : a.k) + at * (KV_B * a.d);
        where = reinterpret_cast<float *>(a.scales + at) + tensor;
        return true;
    };

    // ALL: every token of the block is new
    const auto keys = [&](auto all) {
        constexpr bool ALL = decltype(all)::value;
        const auto is_new = [&](int t) { return ALL || (t0 + t >= start && t0 + t < end); };
        constexpr int W = 2 * WORDS8<T>;
        uint32_t v[NU][W];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = a.by_chunks.div(q), w = q - t * nc;
#pragma unroll
            for (int j = 0; j < W; ++j) v[i][j] = 0;
            if (t < KV_B && is_new(t)) {
                load8(x + (int64_t)t * src.token + 16 * w, src.wide, v[i]);
                load8(x + (int64_t)t * src.token + 16 * w + 8, src.wide, v[i] + W / 2);
            }
        }
        if (!find()) return;
        const float old = holds ? *where : 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) top = larger<T>(top, v[i][j]);
        const BlockScale bs = block_scale<T>(top, old, [&] {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float y = fabsf(value<T>(v[i], j));
                    m = y < INFINITY ? fmaxf(m, y) : m;
                }
            return m;
        });
        __syncwarp();
        if (lane == 0) *where = bs.s;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = a.by_chunks.div(q), w = q - t * nc;
            if (t >= KV_B) continue;
            uint4 *p = reinterpret_cast<uint4 *>(codes + w * 256 + t * 16);
            if (is_new(t)) {
                uint32_t c[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    c[j] = codes4(value<T>(v[i], 4 * j), value<T>(v[i], 4 * j + 1), value<T>(v[i], 4 * j + 2),
                                  value<T>(v[i], 4 * j + 3), bs.s, bs.inv, bs.quick);
                *p = make_uint4(c[0], c[1], c[2], c[3]);
            } else if (t0 + t < start && bs.ratio != 1.0f) {
                const uint4 c = *p;
                *p = make_uint4(rescale4(c.x, bs.ratio), rescale4(c.y, bs.ratio), rescale4(c.z, bs.ratio),
                                rescale4(c.w, bs.ratio));
            }
        }
    };
    const auto values = [&](auto all) {
        constexpr bool ALL = decltype(all)::value;
        const auto is_new = [&](int t) { return ALL || (t0 + t >= start && t0 + t < end); };
        constexpr int NV = (NU + 1) / 2, W = WORDS8<T>;
        uint32_t v[NV][4][W];
        const int last = a.d / 2;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = lane + 32 * i, c = q & 3, e = q >> 2;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1) + 8 * (k >> 1);
#pragma unroll
                for (int j = 0; j < W; ++j) v[i][k][j] = 0;
                if (q < last && is_new(t)) load8(x + (int64_t)t * src.token + 8 * e, src.wide, v[i][k]);
            }
        }
        if (!find()) return;
        const float old = holds ? *where : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < W; ++j) top = larger<T>(top, v[i][k][j]);
        const BlockScale bs = block_scale<T>(top, old, [&] {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float y = fabsf(value<T>(v[i][k], j));
                        m = y < INFINITY ? fmaxf(m, y) : m;
                    }
            return m;
        });
        __syncwarp();
        if (lane == 0) *where = bs.s;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = lane + 32 * i, c = q & 3, e = q >> 2;
            if (q >= last) continue;
            uint32_t fresh = 0, held = 0;  // bytes of new tokens, of tokens from before
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1) + 8 * (k >> 1);
                if (is_new(t)) fresh |= 0xffu << (8 * k);
                if (!ALL && t0 + t < start) held |= 0xffu << (8 * k);
            }
            if (!ALL && !fresh && (!held || bs.ratio == 1.0f)) continue;
            uint32_t *p = reinterpret_cast<uint32_t *>(codes + 8 * e * 16 + 4 * c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t w = codes4(value<T>(v[i][0], j), value<T>(v[i][1], j), value<T>(v[i][2], j), value<T>(v[i][3], j),
                                    bs.s, bs.inv, bs.quick);
                if (!ALL && fresh != 0xffffffffu) {
                    const uint32_t was = p[4 * j];
                    const uint32_t kept = bs.ratio != 1.0f ? rescale4(was, bs.ratio) : was;
                    w = (w & fresh) | (kept & held) | (was & ~(fresh | held));
                }
                p[4 * j] = w;
            }
        }
    };
    if (tensor == 0) full ? keys(std::true_type{}) : keys(std::false_type{});
    else full ? values(std::true_type{}) : values(std::false_type{});
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

#define KV_BY_TYPE(KERNEL, NU)                                                                              \
    do {                                                                                                    \
        if (dtype == SKM_DTYPE_F32) KERNEL<float, NU><<<grid, WARPS * 32, 0, st>>>(a);      \
        else if (dtype == SKM_DTYPE_BF16)                                                                   \
            KERNEL<__nv_bfloat16, NU><<<grid, WARPS * 32, 0, st>>>(a);                   \
        else KERNEL<__half, NU><<<grid, WARPS * 32, 0, st>>>(a);                         \
    } while (0)

static KvCacheArgs with_divisions(KvCacheArgs a) {
    a.by_heads = FastDiv(a.heads);
    a.by_bpp = FastDiv(a.bpp);
    a.by_most = FastDiv(most_blocks_of(a));
    a.by_chunks = FastDiv(a.d / KV_B);
    return a;
}

cudaError_t launch_kv_write(const KvCacheArgs &args, int dtype, cudaStream_t st) {
    const KvCacheArgs a = with_divisions(args);
    const unsigned grid = (unsigned)grid_of(a);
    if (a.d <= 64) KV_BY_TYPE(kv_write_kernel, 2);
    else if (a.d <= 128) KV_BY_TYPE(kv_write_kernel, 4);
    else KV_BY_TYPE(kv_write_kernel, 8);
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
