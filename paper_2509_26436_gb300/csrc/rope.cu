// Rotary positions for sm_103a: y = rotation of x [tokens, heads, dim] by
// position times frequency, pairs (i, i + rotary/2) or (2i, 2i + 1).
//
// HBM-bound: x is read and y written once, 3 operations per element.  A thread
// turns V pairs of one token (two V-element vectors) in several heads, the next
// head's loads under way; the threads of a CTA that have the same pairs in other
// heads share the angles, computed once per CTA, which costs about as much as
// turning them in ten heads.  8192 x 32 x 128 bf16, of a strided tensor: 23.7 us,
// 84% of the copy rate, with 1280 threads per SM (48 registers, the angles read
// from shared memory for each head); 1024 26.1, 1536 24.6; one head in flight
// 24.8; angles in registers as well 26.6; angles per thread 28.5.
#include "quartz_internal.h"
#include "rope.cuh"

namespace quartz {
namespace {

constexpr int kThreads = 128;

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

template <typename T, int V>
__device__ __forceinline__ void store_rounded(T *to, const float (&f)[V])
{
    Vec<T, V> v;
    if constexpr (sizeof(T) == 2 && V > 1) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) w[j] = pack_pair<T>(f[2 * j], f[2 * j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v.e[j] = from_f32<T>(f[j]);
    }
    *reinterpret_cast<Vec<T, V> *>(to) = v;
}

// n / pieces by a product with 2^64 / pieces, rounded up (0: pieces is 1): exact
// for n pieces < 2^64, and places are below 2^40.  (A 64-bit division is some
// hundred instructions.)
__device__ __forceinline__ int64_t token_of(int64_t n, uint64_t inverse)
{
    return inverse ? static_cast<int64_t>(__umul64hi(static_cast<uint64_t>(n), inverse)) : n;
}

// Piece p < pairs / V of a head turns V pairs, the others copy V elements each
// from `rotary` on.  `here` (token, piece) places per CTA, as consecutive
// threads; the threads behind them: the same places in further heads.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 10) rope_kernel(RopeArgs a, int64_t places, uint64_t inverse, int here,
                                                            int heads_each)
{
    griddep_wait();
    __shared__ float2 s_cs[V * kThreads];  // [pair of the piece][place]
    const int pairs = a.rope.rotary / 2;
    const int turns = pairs / V, pieces = turns + (a.dim - a.rope.rotary) / V;
    const int64_t first_place = static_cast<int64_t>(blockIdx.x) * here;
    const int group = threadIdx.x / here, place = threadIdx.x - group * here;
    const int64_t id = first_place + place;
    const bool in = id < places;
    const int64_t t = in ? token_of(id, inverse) : 0;
    const int p = in ? static_cast<int>(id - t * pieces) : 0;
    const bool turn = p < turns;
    const int first = turn ? (a.rope.interleaved ? 2 * p * V : p * V) : a.rope.rotary + (p - turns) * V;
    const int gap = a.rope.interleaved ? V : pairs;  // from the first vector to the second
    const int h0 = group * heads_each, h1 = in ? min(a.heads, h0 + heads_each) : 0;
    const T *x = static_cast<const T *>(a.x) + t * a.x_st + first;
    T *y = static_cast<T *>(a.y) + t * a.y_st + first;

    Vec<T, V> u, w;
    if (h0 < h1) {  // the first head's loads, under way meanwhile
        u = *reinterpret_cast<const Vec<T, V> *>(x + h0 * a.x_sh);
        if (turn) w = *reinterpret_cast<const Vec<T, V> *>(x + h0 * a.x_sh + gap);
    }
    // the CTA's tokens' pairs, those whose piece is among its places
    const int64_t token0 = token_of(first_place, inverse), behind = min(first_place + here, places);
    const int its = static_cast<int>(token_of(behind - 1, inverse) - token0) + 1;
    for (int i = threadIdx.x; i < its * pairs; i += kThreads) {
        const int k = i / pairs, j = i - k * pairs;
        const int64_t at = (token0 + k) * pieces + j / V - first_place;
        if (at >= 0 && at < behind - first_place) {
            const float2 cs = rope_cos_sin(a.rope.positions[token0 + k], rope_unit(a.rope.freqs[j]), a.rope.scale);
            s_cs[(j % V) * here + at] = make_float2(cs.x, a.rope.backward ? -cs.y : cs.y);
        }
    }
    __syncthreads();
    for (int h = h0; h < h1; ++h) {
        Vec<T, V> u2, w2;
        if (h + 1 < h1) {  // the next head's
            u2 = *reinterpret_cast<const Vec<T, V> *>(x + (h + 1) * a.x_sh);
            if (turn) w2 = *reinterpret_cast<const Vec<T, V> *>(x + (h + 1) * a.x_sh + gap);
        }
        T *to = y + h * a.y_sh;
        if (turn) {
            float f[2][V];  // the two vectors' elements
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (a.rope.interleaved) {
                    // elements 2j and 2j + 1 of the 2V read
                    const T x1 = 2 * j < V ? u.e[(2 * j) % V] : w.e[(2 * j) % V];
                    const T x2 = 2 * j + 1 < V ? u.e[(2 * j + 1) % V] : w.e[(2 * j + 1) % V];
                    const float2 r = rope_turn(to_f32<T>(x1), to_f32<T>(x2), s_cs[j * here + place]);
                    f[2 * j / V][(2 * j) % V] = r.x;
                    f[(2 * j + 1) / V][(2 * j + 1) % V] = r.y;
                } else {
                    const float2 r = rope_turn(to_f32<T>(u.e[j]), to_f32<T>(w.e[j]), s_cs[j * here + place]);
                    f[0][j] = r.x;
                    f[1][j] = r.y;
                }
            }
            store_rounded<T, V>(to, f[0]);
            store_rounded<T, V>(to + gap, f[1]);
        } else {
            *reinterpret_cast<Vec<T, V> *>(to) = u;
        }
        u = u2, w = w2;
    }
}

template <typename T, int V>
cudaError_t launch_v(const RopeArgs &a, int64_t tokens, cudaStream_t s)
{
    const int pieces = a.rope.rotary / 2 / V + (a.dim - a.rope.rotary) / V;
    const int64_t places = tokens * pieces;
    const uint64_t inverse = pieces > 1 ? ~uint64_t(0) / pieces + 1 : 0;
    // More groups of heads per CTA while there are fewer than 2048 threads per SM
    // (8192 x 32 x 128: 23.7 us; up to 1024 25.6, up to 4096 24.5)
    const int64_t threads = int64_t(device_sms()) * 2048;
    int groups = 1;
    while (groups < 32 && groups < a.heads && places * groups < threads) groups *= 2;
    const int here = kThreads / groups, each = (a.heads + groups - 1) / groups;
    return launch_pdl(rope_kernel<T, V>, dim3(static_cast<unsigned>((places + here - 1) / here)), dim3(kThreads), 0, s, a, places,
                      inverse, here, each);
}

// The widest vectors of V elements (16 bytes, or 8) that sizes, strides and
// addresses allow; else one element at a time.
template <typename T>
bool fits(const RopeArgs &a, int v)
{
    const uintptr_t m = v * sizeof(T) - 1;
    return (a.rope.rotary / 2) % v == 0 && (a.dim - a.rope.rotary) % v == 0 && a.x_st % v == 0 && a.x_sh % v == 0 &&
           a.y_st % v == 0 && a.y_sh % v == 0 && (reinterpret_cast<uintptr_t>(a.x) & m) == 0 &&
           (reinterpret_cast<uintptr_t>(a.y) & m) == 0;
}

template <typename T>
cudaError_t launch_t(const RopeArgs &a, int64_t tokens, cudaStream_t s)
{
    constexpr int wide = 16 / sizeof(T);
    if (fits<T>(a, wide)) return launch_v<T, wide>(a, tokens, s);
    if (fits<T>(a, wide / 2)) return launch_v<T, wide / 2>(a, tokens, s);
    return launch_v<T, 1>(a, tokens, s);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs &a, int64_t tokens, cudaStream_t s)
{
    if (a.type == QUARTZ_OUT_F16) return launch_t<__half>(a, tokens, s);
    if (a.type == QUARTZ_OUT_BF16) return launch_t<__nv_bfloat16>(a, tokens, s);
    return launch_t<float>(a, tokens, s);
}

}  // namespace quartz
