// Rotary positions for sm_103a: y = rotation of x [tokens, heads, dim] by
// position times frequency, pairs (i, i + rotary/2) or (2i, 2i + 1).
//
// HBM-bound: x is read and y written once, 3 operations per element.  A CTA
// goes through tokens; a thread has the same pieces of a head (V pairs each,
// two V-element vectors) in all of them.  The next token's vectors are loaded
// while this one's angles, one per thread, are computed into shared memory and
// its pairs turned.
#include "quartz_internal.h"
#include "rope.cuh"

namespace quartz {
namespace {

constexpr int kMaxPairs = 256;
constexpr int kThreads = 128;

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

// Piece p < pairs / V of a head turns V pairs, the others copy V elements each
// from `rotary` on.  ITEMS pieces per thread; blockIdx.y: further pieces.
template <typename T, int V, int ITEMS>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a, int tokens)
{
    griddep_wait();
    __shared__ float2 s_cs[2][kMaxPairs];
    __shared__ uint64_t s_unit[kMaxPairs];
    const int pairs = a.rope.rotary / 2;
    const int turns = pairs / V, pieces = turns + (a.dim - a.rope.rotary) / V;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.y);
    int64_t in1[ITEMS], out1[ITEMS];
    int gap[ITEMS], cs_at[ITEMS];  // from the first vector to the second (0: none, copy); angles
    bool mine[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int i = (blockIdx.y * ITEMS + k) * kThreads + threadIdx.x;
        const int h = i / pieces, p = i - h * pieces;
        mine[k] = h < a.heads;
        const bool turn = p < turns;
        const int o1 = turn ? (a.rope.interleaved ? 2 * p * V : p * V) : a.rope.rotary + (p - turns) * V;
        gap[k] = turn ? (a.rope.interleaved ? V : pairs) : 0;
        cs_at[k] = turn ? p * V : 0;
        in1[k] = h * a.x_sh + o1;
        out1[k] = h * a.y_sh + o1;
    }
    for (int i = threadIdx.x; i < pairs; i += kThreads) s_unit[i] = rope_unit(a.rope.freqs[i]);
    const float sign = a.rope.backward ? -1.f : 1.f;

    Vec<T, V> u[ITEMS], w[ITEMS];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
            if (mine[k]) {
                const T *p = x + t * a.x_st + in1[k];
                u[k] = *reinterpret_cast<const Vec<T, V> *>(p);
                if (gap[k]) w[k] = *reinterpret_cast<const Vec<T, V> *>(p + gap[k]);
            }
    };
    int64_t t = blockIdx.x;
    int64_t pos = a.rope.positions[t];
    load(t);
    __syncthreads();  // s_unit
    for (int buffer = 0; t < tokens; buffer ^= 1) {
        for (int i = threadIdx.x; i < pairs; i += kThreads) {
            const float2 cs = rope_cos_sin(pos, s_unit[i], a.rope.scale);
            s_cs[buffer][i] = make_float2(cs.x, sign * cs.y);
        }
        const int64_t now = t;
        t += gridDim.x;
        Vec<T, V> cu[ITEMS], cw[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) cu[k] = u[k], cw[k] = w[k];
        if (t < tokens) {
            pos = a.rope.positions[t];
            load(t);
        }
        __syncthreads();  // the angles; the other buffer's readers are past the barrier before
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            if (!mine[k]) continue;
            T *to = y + now * a.y_st + out1[k];
            if (gap[k]) {
                Vec<T, V> r1, r2;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 cs = s_cs[buffer][cs_at[k] + j];
                    if (a.rope.interleaved) {
                        // elements 2j and 2j + 1 of the 2V read
                        const T x1 = 2 * j < V ? cu[k].e[(2 * j) % V] : cw[k].e[(2 * j) % V];
                        const T x2 = 2 * j + 1 < V ? cu[k].e[(2 * j + 1) % V] : cw[k].e[(2 * j + 1) % V];
                        const float2 r = rope_turn(to_f32<T>(x1), to_f32<T>(x2), cs);
                        (2 * j < V ? r1 : r2).e[(2 * j) % V] = from_f32<T>(r.x);
                        (2 * j + 1 < V ? r1 : r2).e[(2 * j + 1) % V] = from_f32<T>(r.y);
                    } else {
                        const float2 r = rope_turn(to_f32<T>(cu[k].e[j]), to_f32<T>(cw[k].e[j]), cs);
                        r1.e[j] = from_f32<T>(r.x);
                        r2.e[j] = from_f32<T>(r.y);
                    }
                }
                *reinterpret_cast<Vec<T, V> *>(to) = r1;
                *reinterpret_cast<Vec<T, V> *>(to + gap[k]) = r2;
            } else {
                *reinterpret_cast<Vec<T, V> *>(to) = cu[k];
            }
        }
    }
}

template <typename T, int V, int ITEMS>
cudaError_t launch_items(const RopeArgs &a, int64_t tokens, int64_t items, cudaStream_t s)
{
    const int64_t y = (items + ITEMS * kThreads - 1) / (ITEMS * kThreads);
    int64_t x = (152 * 16 + y - 1) / y;  // some 16 CTAs per SM, each with several tokens where there are more
    if (x > tokens) x = tokens;
    return launch_pdl(rope_kernel<T, V, ITEMS>, dim3(static_cast<unsigned>(x), static_cast<unsigned>(y)), dim3(kThreads), 0, s, a,
                      static_cast<int>(tokens));
}

template <typename T, int V>
cudaError_t launch_v(const RopeArgs &a, int64_t tokens, cudaStream_t s)
{
    const int64_t items = static_cast<int64_t>(a.heads) * (a.rope.rotary / 2 / V + (a.dim - a.rope.rotary) / V);
    // Two pieces per thread share a CTA's angles where there is work for all
    // SMs; else one.
    if (tokens * items >= 152 * 2048) return launch_items<T, V, 2>(a, tokens, items, s);
    return launch_items<T, V, 1>(a, tokens, items, s);
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
