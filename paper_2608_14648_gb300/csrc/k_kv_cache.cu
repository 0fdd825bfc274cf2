// Writing keys and values into the 8-bit cache and reading them back.
//
// One warp takes one block (16 tokens) of one head's keys or values: it holds
// the block's new values in registers, so the largest magnitude, the scale and
// the codes come from one read of the input.  Both kernels move bytes and
// nothing else bounds them; a warp needs no other warp, so an append (one
// token, a warp busy for its memory latencies) and a prompt (thousands of
// independent 4 KB reads in flight) are the same code.
//
// Lanes: keys, a unit is 16 dims of a token (a 16-byte code store, two 16-byte
// loads of 16-bit values), consecutive lanes along d; values, whose blocks
// keep the 16 tokens of a dim together, a unit is 8 dims of the four tokens
// that share a 32-bit word, so the transposition stays in registers.
//
// Rounding: code = rint(x / scale) with the quotient rounded to fp32.  x times
// the reciprocal is within 1.6e-5 of x / scale (|quotient| < 128, two roundings
// of 2^-24 relative), the fp32 quotient within 8e-6, so both round to the same
// integer unless x times the reciprocal lies within 1e-4 of a half; only those
// elements (and infinities and NaN) take the division.
#include <type_traits>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int WARPS = 8;
constexpr float CODE_MAGIC = 12583040.0f;  // 1.5 2^23 + 128: q + this holds rint(q) + 128 in its low byte
constexpr float NEAR_HALF = 0.4999f;

// 8 consecutive values
template <typename T>
__device__ __forceinline__ void load8(const T *p, int wide, float *v) {
    if (!wide) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)p[i];
        return;
    }
    if constexpr (std::is_same<T, float>::value) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                v[2 * i] = f.x, v[2 * i + 1] = f.y;
            } else {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
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

__device__ __forceinline__ float warp_max(float m) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

__device__ __noinline__ uint32_t code_exact(float x, float s) {
    float q = __fdiv_rn(x, s);
    q = q == q ? fminf(fmaxf(rintf(q), -127.0f), 127.0f) : 0.0f;
    return (uint32_t)(int)(q + 128.0f);
}

// codes of four values in a word, the first in the low byte; quick: the
// reciprocal of s is a normal number
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float s, float inv, bool quick) {
    const float fa = fmaf(a, inv, CODE_MAGIC), fb = fmaf(b, inv, CODE_MAGIC);
    const float fc = fmaf(c, inv, CODE_MAGIC), fd = fmaf(d, inv, CODE_MAGIC);
    const float ra = fmaf(a, inv, CODE_MAGIC - fa), rb = fmaf(b, inv, CODE_MAGIC - fb);
    const float rc = fmaf(c, inv, CODE_MAGIC - fc), rd = fmaf(d, inv, CODE_MAGIC - fd);
    const float far = fmaxf(fmaxf(fabsf(ra), fabsf(rb)), fmaxf(fabsf(rc), fabsf(rd)));
    const bool fine = quick && far <= NEAR_HALF && ra == ra && rb == rb && rc == rc && rd == rd;
    if (fine) {
        const uint32_t lo = __byte_perm(__float_as_uint(fa), __float_as_uint(fb), 0x0040);
        const uint32_t hi = __byte_perm(__float_as_uint(fc), __float_as_uint(fd), 0x0040);
        return __byte_perm(lo, hi, 0x5410);
    }
    return code_exact(a, s) | code_exact(b, s) << 8 | code_exact(c, s) << 16 | code_exact(d, s) << 24;
}

// codes of a word of the block's earlier tokens after its scale grew by 1 / r
__device__ __forceinline__ uint32_t rescale4(uint32_t word, float r) {
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) out |= (uint32_t)(int)(rintf(kv_code(word, i) * r) + 128.0f) << (8 * i);
    return out;
}

// The block's scale and what it was: a = the lanes' largest |x| with
// infinities counted, fine(): the largest finite one (rare)
struct BlockScale {
    float s, inv, ratio;  // ratio: old / s, 1 when the codes held stay as they are
    bool quick;
};
template <typename Fine>
__device__ __forceinline__ BlockScale block_scale(float a, float *where, bool holds, int lane, Fine fine) {
    a = warp_max(a);
    if (a == INFINITY) a = warp_max(fine());
    const float old = holds ? *where : 0.0f;
    __syncwarp();
    BlockScale b;
    b.s = fmaxf(old, a * (1.0f / 127.0f));
    b.ratio = old > 0.0f && b.s > old ? __fdiv_rn(old, b.s) : 1.0f;
    b.quick = b.s > 1e-37f;
    b.inv = b.quick ? __frcp_rn(b.s) : 0.0f;
    if (lane == 0) *where = b.s;
    return b;
}

// Warps: one a (sequence, block its new rows reach, head, tensor).  NU: units a lane.
template <typename T, int NU>
__global__ void __launch_bounds__(WARPS * 32) kv_write_kernel(KvCacheArgs a, int most_blocks) {
    const int lane = threadIdx.x & 31;
    int64_t u = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
    const int tensor = (int)(u & 1);
    u >>= 1;
    const int h = (int)(u % a.heads);
    u /= a.heads;
    const int b = (int)(u / most_blocks);
    if (b >= a.batch) return;
    const int2 rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
    const int start = max(a.pos[b], 0);
    const int cap = a.cols * a.page;
    const int end = (int)min((int64_t)start + rows.y, (int64_t)cap);
    const int blk = start / KV_B + (int)(u % most_blocks);
    const int t0 = blk * KV_B;
    if (t0 >= end) return;
    const int pg = a.table[(int64_t)b * a.cols + blk / a.bpp];
    if (pg < 0 || pg >= a.pages) return;
    const int64_t at = ((int64_t)pg * a.heads + h) * a.bpp + blk % a.bpp;
    const int nc = a.d / KV_B;
    const KvTokens src = tensor ? a.V : a.K;
    const T *x = static_cast<const T *>(src.x) + (int64_t)(rows.x - start + t0) * src.token + (int64_t)h * src.head;
    uint8_t *codes = (tensor ? a.v : a.k) + at * (KV_B * a.d);
    float *where = reinterpret_cast<float *>(a.scales + at) + tensor;
    const bool holds = start > t0;
    // tokens of the block that are new / held from before
    const auto is_new = [&](int t) { return t0 + t >= start && t0 + t < end; };
    float top = 0.0f;

    if (tensor == 0) {
        float v[NU][16];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = q / nc, w = q - t * nc;
            if (t < KV_B && is_new(t)) {
                load8(x + (int64_t)t * src.token + 16 * w, src.wide, v[i]);
                load8(x + (int64_t)t * src.token + 16 * w + 8, src.wide, v[i] + 8);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) v[i][j] = 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(v[i][j]));
        const BlockScale bs = block_scale(top, where, holds, lane, [&] {
            float m = 0.0f;
            for (int i = 0; i < NU; ++i)
                for (int j = 0; j < 16; ++j) m = fmaxf(m, fabsf(v[i][j]) < INFINITY ? fabsf(v[i][j]) : 0.0f);
            return m;
        });
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = q / nc, w = q - t * nc;
            if (t >= KV_B) continue;
            uint4 *p = reinterpret_cast<uint4 *>(codes + w * 256 + t * 16);
            if (is_new(t)) {
                uint32_t c[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    c[j] = bs.s > 0.0f ? codes4(v[i][4 * j], v[i][4 * j + 1], v[i][4 * j + 2], v[i][4 * j + 3], bs.s,
                                                bs.inv, bs.quick)
                                       : 0x80808080u;
                *p = make_uint4(c[0], c[1], c[2], c[3]);
            } else if (t0 + t < start && bs.ratio != 1.0f) {
                const uint4 c = *p;
                *p = make_uint4(rescale4(c.x, bs.ratio), rescale4(c.y, bs.ratio), rescale4(c.z, bs.ratio),
                                rescale4(c.w, bs.ratio));
            }
        }
    } else {
        constexpr int NV = (NU + 1) / 2;
        float v[NV][4][8];
        const int last = a.d / 2;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = lane + 32 * i, c = q & 3, e = q >> 2;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1) + 8 * (k >> 1);
                if (q < last && is_new(t)) {
                    load8(x + (int64_t)t * src.token + 8 * e, src.wide, v[i][k]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][k][j] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[i][k][j]));
        const BlockScale bs = block_scale(top, where, holds, lane, [&] {
            float m = 0.0f;
            for (int i = 0; i < NV; ++i)
                for (int k = 0; k < 4; ++k)
                    for (int j = 0; j < 8; ++j)
                        m = fmaxf(m, fabsf(v[i][k][j]) < INFINITY ? fabsf(v[i][k][j]) : 0.0f);
            return m;
        });
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int q = lane + 32 * i, c = q & 3, e = q >> 2;
            if (q >= last) continue;
            uint32_t fresh = 0, held = 0;  // bytes of new tokens, of tokens from before
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1) + 8 * (k >> 1);
                if (is_new(t)) fresh |= 0xffu << (8 * k);
                if (t0 + t < start) held |= 0xffu << (8 * k);
            }
            if (!fresh && (!held || bs.ratio == 1.0f)) continue;
            uint32_t *p = reinterpret_cast<uint32_t *>(codes + 8 * e * 16 + 4 * c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t w = bs.s > 0.0f
                                 ? codes4(v[i][0][j], v[i][1][j], v[i][2][j], v[i][3][j], bs.s, bs.inv, bs.quick)
                                 : 0x80808080u;
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
__global__ void __launch_bounds__(WARPS * 32) kv_read_kernel(KvCacheArgs a, int most_blocks) {
    const int lane = threadIdx.x & 31;
    int64_t u = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
    const int tensor = (int)(u & 1);
    u >>= 1;
    const int h = (int)(u % a.heads);
    u /= a.heads;
    const int b = (int)(u / most_blocks);
    if (b >= a.batch) return;
    T *dst = static_cast<T *>(tensor ? a.outv : a.outk);
    if (!dst) return;
    const int2 rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
    const int start = max(a.pos[b], 0);
    const int64_t end = (int64_t)start + rows.y;
    const int64_t blk = start / KV_B + u % most_blocks;
    const int64_t t0 = blk * KV_B;
    if (t0 >= end) return;
    const int64_t col = blk / a.bpp;
    const int pg = col < a.cols ? a.table[(int64_t)b * a.cols + col] : -1;
    const bool there = pg >= 0 && pg < a.pages;
    const int64_t at = there ? ((int64_t)pg * a.heads + h) * a.bpp + blk % a.bpp : 0;
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
            const int q = lane + 32 * i, t = q / nc, w = q - t * nc;
            c[i] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
            if (there && t < KV_B && wanted(t)) c[i] = *reinterpret_cast<const uint4 *>(codes + w * 256 + t * 16);
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int q = lane + 32 * i, t = q / nc, w = q - t * nc;
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

int64_t grid_of(const KvCacheArgs &a) {
    return cdiv((int64_t)a.batch * most_blocks_of(a) * a.heads * 2, WARPS);
}

}  // namespace

#define KV_BY_TYPE(KERNEL, NU)                                                                              \
    do {                                                                                                    \
        if (dtype == SKM_DTYPE_F32) KERNEL<float, NU><<<grid, WARPS * 32, 0, st>>>(a, most_blocks_of(a));      \
        else if (dtype == SKM_DTYPE_BF16)                                                                   \
            KERNEL<__nv_bfloat16, NU><<<grid, WARPS * 32, 0, st>>>(a, most_blocks_of(a));                   \
        else KERNEL<__half, NU><<<grid, WARPS * 32, 0, st>>>(a, most_blocks_of(a));                         \
    } while (0)

cudaError_t launch_kv_write(const KvCacheArgs &a, int dtype, cudaStream_t st) {
    const unsigned grid = (unsigned)grid_of(a);
    if (a.d <= 64) KV_BY_TYPE(kv_write_kernel, 2);
    else if (a.d <= 128) KV_BY_TYPE(kv_write_kernel, 4);
    else KV_BY_TYPE(kv_write_kernel, 8);
    return launched();
}

cudaError_t launch_kv_read(const KvCacheArgs &a, int dtype, cudaStream_t st) {
    const unsigned grid = (unsigned)grid_of(a);
    if (a.d <= 64) KV_BY_TYPE(kv_read_kernel, 2);
    else if (a.d <= 128) KV_BY_TYPE(kv_read_kernel, 4);
    else KV_BY_TYPE(kv_read_kernel, 8);
    return launched();
}

}  // namespace skm
