// Rotary positions of query and key rows (Su et al., RoFormer, 2021): the dims of a head form
// pairs, and at position p pair i turns by the angle a = p f_i:
//   y1 = g (x1 cos a - x2 sin a),  y2 = g (x1 sin a + x2 cos a);  transposed: -a, for gradients.
//
// The angle.  Frequencies are turns a position in 64-bit fixed point, so p f mod 1 is one integer
// product that wraps where the circle does, exact at every position; the nearest quarter turn comes off
// as an integer too, and sincospi sees at most an eighth of a turn.
//
// A CTA takes the rows of a few tokens: first their angles, a sine and a cosine a pair and token to
// shared memory (one a thread where there are that many), then heads and vectors, all with the same angles.  Work is
// cut finer, by heads, where there are few tokens.
//
// What bounds it is HBM, a value is read and written once, and what keeps it from that are reads in flight and instructions.
// Gradients of 12 prompts of up to 2500 tokens, 40 heads of 128 dims, 64 of them turned, bf16: 60 us, 84% of a copy's rate
// (CTAs of 256 threads 66, two rows at a time 66, both 68, eight rows 65; a vector as words 72 -> 68 and 77 -> 72 before).
#include <algorithm>
#include <type_traits>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int THREADS = 128, TOKENS_MOST = 16, AT_ONCE = 4;  // AT_ONCE: rows that a thread reads before it uses the first

// The sequence that row `tok` belongs to, -1 for none: the last of cu[0 .. batch] that is
// not above it.  By a whole warp, four entries a lane and round.
__device__ __forceinline__ int sequence_of(const int32_t *cu, int batch, int tok, int lane) {
    int lo = 0, n = batch + 1;  // the last one not above lies in [lo, lo + n), if anywhere
    for (;;) {
        const int step = (n + 127) / 128;
        int below = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t i = (int64_t)(lane + 32 * k) * step;
            const bool is = i < n && cu[lo + i] <= tok;
            below += __popc(__ballot_sync(0xffffffffu, is));
        }
        if (below == 0) return -1;
        const int skip = (below - 1) * step;
        lo += skip;
        n = min(step, n - skip);
        if (step == 1) break;
    }
    return lo < batch ? lo : -1;
}

// V elements as words (one 16-bit element: in a word's low half)
template <typename T, int V>
constexpr int WORDS = sizeof(T) * V < 4 ? 1 : sizeof(T) * V / 4;
template <typename T, int V>
__device__ __forceinline__ void load_words(const T *x, uint32_t *w) {
    constexpr int BYTES = sizeof(T) * V;
    if constexpr (BYTES == 2) {
        w[0] = *reinterpret_cast<const uint16_t *>(x);
    } else if constexpr (BYTES == 4) {
        w[0] = *reinterpret_cast<const uint32_t *>(x);
    } else if constexpr (BYTES == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(x);
        w[0] = v.x, w[1] = v.y;
    } else {
        static_assert(BYTES == 16);
        const uint4 v = *reinterpret_cast<const uint4 *>(x);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_words(T *y, const uint32_t *w) {
    constexpr int BYTES = sizeof(T) * V;
    if constexpr (BYTES == 2) *reinterpret_cast<uint16_t *>(y) = (uint16_t)w[0];
    else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t *>(y) = w[0];
    else if constexpr (BYTES == 8) *reinterpret_cast<uint2 *>(y) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint4 *>(y) = make_uint4(w[0], w[1], w[2], w[3]);
}
// elements 2 i and 2 i + 1 (of one element: it and anything)
template <typename T>
__device__ __forceinline__ float2 two_of(const uint32_t *w, int i) {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2 *>(w + i));
    else return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
template <typename T>
__device__ __forceinline__ void put_two(uint32_t *w, int i, float2 v) {
    if constexpr (sizeof(T) == 4) {
        w[2 * i] = __float_as_uint(v.x), w[2 * i + 1] = __float_as_uint(v.y);
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(v.x, v.y);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
}

// What a thread takes of a row: a vector of V elements, neighbours in pairs (NEXT; with V = 1 two elements, one at a time), or one
// of each half of the dims
template <typename T, int V, bool NEXT>
struct Unit {
    static constexpr int E = NEXT && V == 1 ? 2 : V, N = (E + 1) / 2;  // elements of p, twos of them
    uint32_t p[N * 2 * sizeof(T) / 4], q[N * 2 * sizeof(T) / 4];
    __device__ __forceinline__ void load(const T *x, int half, bool copy) {
        if constexpr (E > V) {
            uint32_t a[1], b[1] = {0};
            load_words<T, 1>(x, a);
            if (!copy) load_words<T, 1>(x + 1, b);
            if constexpr (sizeof(T) == 4) p[0] = a[0], p[1] = b[0];
            else p[0] = a[0] | b[0] << 16;
        } else {
            load_words<T, V>(x, p);
            if constexpr (!NEXT)
                if (!copy) load_words<T, V>(x + half, q);
        }
    }
    __device__ __forceinline__ void store(T *y, int half, bool copy) const {
        if constexpr (E > V) {
            const uint32_t b = sizeof(T) == 4 ? p[sizeof(T) / 4] : p[0] >> 16;
            store_words<T, 1>(y, p);
            if (!copy) store_words<T, 1>(y + 1, &b);
        } else {
            store_words<T, V>(y, p);
            if constexpr (!NEXT)
                if (!copy) store_words<T, V>(y + half, q);
        }
    }
    __device__ __forceinline__ void turn(const float2 *cs) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float2 a = two_of<T>(p, i);
            if constexpr (NEXT) {
                const float2 r = cs[i];
                put_two<T>(p, i, make_float2(a.x * r.x - a.y * r.y, a.x * r.y + a.y * r.x));
            } else {
                const float2 b = two_of<T>(q, i);
                // (cosine, sine) of two pairs at once: an even number of pairs from an even one on
                const float4 r = E > 1 ? *reinterpret_cast<const float4 *>(cs + 2 * i) : make_float4(cs[0].x, cs[0].y, 0.0f, 0.0f);
                put_two<T>(p, i, make_float2(a.x * r.x - b.x * r.y, a.y * r.z - b.y * r.w));
                put_two<T>(q, i, make_float2(a.x * r.y + b.x * r.x, a.y * r.w + b.y * r.z));
            }
        }
    }
};

// V: elements of a vector
template <typename T, int V, bool NEXT>
__global__ void __launch_bounds__(THREADS) rotary_kernel(const __grid_constant__ RotaryArgs a) {
    extern __shared__ __align__(16) float2 angles[];  // [tokens][dims / 2] cosine, sine
    __shared__ int there[TOKENS_MOST];
    const int tid = threadIdx.x, lane = tid & 31, half = a.dims / 2;
    const int tok0 = blockIdx.x / a.cuts * a.tile, cut = blockIdx.x % a.cuts, nt = min(a.tile, a.tokens - tok0);
    __shared__ int64_t at[TOKENS_MOST];
    bool mine = true;
    for (int i = tid >> 5; i < nt; i += THREADS / 32) {
        const int b = sequence_of(a.cu, a.batch, tok0 + i, lane);
        int2 rows = make_int2(0, 0);
        if (b >= 0) rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
        const bool in = tok0 + i >= rows.x && tok0 + i < rows.x + rows.y;
        mine = mine && in;
        if (lane == 0) {
            there[i] = in;
            if (in) at[i] = (int64_t)a.pos[b] + (tok0 + i - rows.x);
        }
    }
    const bool all = __syncthreads_and(mine);  // (rows that belong to no sequence are left alone)
    for (int i = tid; i < nt * half; i += THREADS) {
        const int t = a.by_half.div(i), pair = i - t * half;
        if (!there[t]) continue;
        const uint64_t turn = (uint64_t)at[t] * a.turns[pair];
        const uint32_t quarter = (uint32_t)((turn + (uint64_t(1) << 61)) >> 62) & 3u;
        const int64_t rest = (int64_t)(turn - ((uint64_t)quarter << 62));
        float s, c;
        sincospif((float)rest * 1.0842022e-19f, &s, &c);  // 2^-63
        const float c1 = quarter & 1 ? s : c, s1 = quarter & 1 ? c : s;
        // quarters 1 and 2 have a negative cosine, 2 and 3 a negative sine
        angles[i] = make_float2((quarter == 1 || quarter == 2) ? -c1 * a.gain : c1 * a.gain, quarter >= 2 ? -s1 * a.sine : s1 * a.sine);
    }
    __syncthreads();
    // units: per token and head the vectors of a rotated head (NEXT: pairs of neighbours, a vector a
    // unit; else a vector of the first half and one of the second), then those copied.  A thread keeps to one unit
    // and goes from row to row (token, head), so that its addresses are additions
    constexpr int E = Unit<T, V, NEXT>::E;
    const int turned = NEXT ? a.dims / E : half / V, units = turned + a.copied / V;
    const int step = max(THREADS / units, 1), first = a.by_units.div(tid);
    if (units <= THREADS && first >= step) return;
    for (int u = tid - (units <= THREADS ? first * units : 0); u < units; u += THREADS) {
        const bool copy = u >= turned;
        const int dim = copy ? a.dims + (u - turned) * V : u * E;
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
            const RotaryPart &part = a.part[k];
            const int h0 = part.heads * cut / a.cuts, nh = part.heads * (cut + 1) / a.cuts - h0;
            if (nh == 0) continue;
            int row = units <= THREADS ? first : 0, t = row / nh, head = row - t * nh;
            const T *x = static_cast<const T *>(part.x) + (int64_t)(tok0 + t) * part.x_token + (int64_t)(h0 + head) * part.x_head + dim;
            T *y = static_cast<T *>(part.y) + (int64_t)(tok0 + t) * part.y_token + (int64_t)(h0 + head) * part.y_head + dim;
            const int64_t x_step = step * part.x_head, y_step = step * part.y_head;
            const int64_t x_wrap = part.x_token - nh * part.x_head, y_wrap = part.y_token - nh * part.y_head;
            // a few rows at a time: all are read before one is used
            while (t < nt) {
                Unit<T, V, NEXT> unit[AT_ONCE];
                T *to[AT_ONCE];
                int of[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    to[i] = y;
                    of[i] = t < nt && (all || there[t]) ? t : -1;
                    if (of[i] >= 0) unit[i].load(x, half, copy);
                    head += step, x += x_step, y += y_step;
                    while (head >= nh) head -= nh, x += x_wrap, y += y_wrap, ++t;
                }
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    if (of[i] < 0) continue;
                    if (!copy) unit[i].turn(angles + of[i] * half + (NEXT ? dim / 2 : dim));
                    unit[i].store(to[i], half, copy);
                }
            }
        }
    }
}

template <typename T, int V, bool NEXT>
cudaError_t run(RotaryArgs a, cudaStream_t st) {
    const int half = a.dims / 2;
    // as many tokens a CTA as there are angles for its threads, as long as all SMs have CTAs
    a.tile = std::max(1, std::min({THREADS / half, TOKENS_MOST, a.tokens / (4 * KV_SMS)}));
    a.cuts = (int)std::max<int64_t>(1, std::min<int64_t>(a.heads, 2 * KV_SMS / a.tokens));
    a.by_half = FastDiv(half);
    a.by_units = FastDiv((NEXT ? a.dims / (V == 1 ? 2 : V) : half / V) + a.copied / V);
    const int64_t grid = cdiv(a.tokens, a.tile) * a.cuts;
    rotary_kernel<T, V, NEXT><<<(unsigned)grid, THREADS, (size_t)a.tile * half * sizeof(float2), st>>>(a);
    return launched();
}
template <typename T, int V>
cudaError_t run(const RotaryArgs &a, cudaStream_t st) {
    return a.interleaved ? run<T, V, true>(a, st) : run<T, V, false>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs &a, int dtype, int vec, cudaStream_t st) {
    if (dtype == SKM_DTYPE_F32) return vec >= 4 ? run<float, 4>(a, st) : vec >= 2 ? run<float, 2>(a, st) : run<float, 1>(a, st);
    if (dtype == SKM_DTYPE_BF16)
        return vec >= 8 ? run<__nv_bfloat16, 8>(a, st) : vec >= 2 ? run<__nv_bfloat16, 2>(a, st) : run<__nv_bfloat16, 1>(a, st);
    return vec >= 8 ? run<__half, 8>(a, st) : vec >= 2 ? run<__half, 2>(a, st) : run<__half, 1>(a, st);
}

}  // namespace skm
