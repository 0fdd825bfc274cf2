// Rotary positions of query and key rows (Su et al., RoFormer, 2021): the dims of a head form
// pairs, and at position p pair i turns by the angle a = p f_i:
//   y1 = g (x1 cos a - x2 sin a),  y2 = g (x1 sin a + x2 cos a);  transposed: -a, for gradients.
//
// The angle.  Frequencies are turns a position in 64-bit fixed point, so p f mod 1 is one integer
// product that wraps where the circle does, exact at every position; the nearest quarter turn comes off
// as an integer too, and sincospi sees at most an eighth of a turn.
//
// A CTA takes the rows of a few tokens: first their angles, a sine and a cosine a pair and token to
// shared memory (one a thread where there are 256), then heads and vectors, all with the same angles.  Work is
// cut finer, by heads, where there are few tokens.  What bounds it is HBM: a value is read and written once.
#include <algorithm>
#include <type_traits>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int THREADS = 256, TOKENS_MOST = 16;

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

template <typename T>
__device__ __forceinline__ float as_float(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else if constexpr (std::is_same<T, __half>::value) return __half2float(x);
    else return __bfloat162float(x);
}
template <typename T>
__device__ __forceinline__ T as_type(float x) {
    if constexpr (sizeof(T) == 4) return x;
    else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

// A vector of neighbours (NEXT), or one of each half of the dims
template <typename T, int E, int V, bool NEXT>
struct Unit {
    Vec<T, E> p, q;
    __device__ __forceinline__ void load(const T *x, int half, bool copy) {
#pragma unroll
        for (int k = 0; k < E; k += V)
            if (k == 0 || !copy) *reinterpret_cast<Vec<T, V> *>(p.v + k) = *reinterpret_cast<const Vec<T, V> *>(x + k);
        if (!NEXT && !copy) q = *reinterpret_cast<const Vec<T, E> *>(x + half);
    }
    __device__ __forceinline__ void store(T *y, int half, bool copy) const {
#pragma unroll
        for (int k = 0; k < E; k += V)
            if (k == 0 || !copy) *reinterpret_cast<Vec<T, V> *>(y + k) = *reinterpret_cast<const Vec<T, V> *>(p.v + k);
        if (!NEXT && !copy) *reinterpret_cast<Vec<T, E> *>(y + half) = q;
    }
    __device__ __forceinline__ void turn(const float2 *cs) {
        constexpr int N = NEXT ? E / 2 : E;  // pairs; their angles two at a time (an even number from an even one on)
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            const float4 two = N > 1 ? *reinterpret_cast<const float4 *>(cs + k) : make_float4(cs[k].x, cs[k].y, 0.0f, 0.0f);
#pragma unroll
            for (int i = k; i < k + 2 && i < N; ++i) {
                const float2 one = i == k ? make_float2(two.x, two.y) : make_float2(two.z, two.w);
                if constexpr (NEXT) pair(p.v[2 * i], p.v[2 * i + 1], one);
                else pair(p.v[i], q.v[i], one);
            }
        }
    }
    __device__ __forceinline__ static void pair(T &x1, T &x2, float2 cs) {
        const float a = as_float(x1), b = as_float(x2);
        x1 = as_type<T>(a * cs.x - b * cs.y);
        x2 = as_type<T>(a * cs.y + b * cs.x);
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
    for (int i = tid >> 5; i < nt; i += THREADS / 32) {
        const int b = sequence_of(a.cu, a.batch, tok0 + i, lane);
        if (lane == 0) {
            bool in = false;
            if (b >= 0) {
                const int2 rows = kv_rows_of(a.cu, b, a.tokens, a.max_tokens);
                in = tok0 + i >= rows.x && tok0 + i < rows.x + rows.y;
                at[i] = (int64_t)a.pos[b] + (tok0 + i - rows.x);
            }
            there[i] = in;
        }
    }
    __syncthreads();
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
    constexpr int E = NEXT && V == 1 ? 2 : V;  // elements of a unit's vector, loaded one at a time where V is 1
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
            // the next row's vectors are read before this one's are used
            Unit<T, E, V, NEXT> now, next;
            bool in = t < nt && there[t];
            if (in) now.load(x, half, copy);
            while (t < nt) {
                const int t_now = t;
                const bool in_now = in;
                T *y_now = y;
                head += step, x += x_step, y += y_step;
                while (head >= nh) head -= nh, x += x_wrap, y += y_wrap, ++t;
                in = t < nt && there[t];
                if (in) next.load(x, half, copy);
                if (in_now) {
                    if (!copy) now.turn(angles + t_now * half + (NEXT ? dim / 2 : dim));
                    now.store(y_now, half, copy);
                }
                now = next;
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
