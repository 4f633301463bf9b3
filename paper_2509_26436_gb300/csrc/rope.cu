// Rotary positions for sm_103a: y = rotation of x [tokens, heads, dim] by
// position times frequency, pairs (i, i + rotary/2) or (2i, 2i + 1).
//
// HBM-bound: x is read and y written once, 3 operations per element.  A CTA
// takes one token and some of its heads.  Its threads first load their pairs
// of up to kHeads heads (two V-element vectors each, all in flight together),
// then compute the token's angles once, one per thread, into shared memory,
// and turn the loaded pairs.
#include "quartz_internal.h"
#include "rope.cuh"

namespace quartz {
namespace {

constexpr int kMaxPairs = 256;
constexpr int kThreadsMax = 256;

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

// blockDim = (pieces of a head, head lanes): piece p < pairs / V turns V pairs,
// the others copy V elements each from `rotary` on.  HEADS heads per thread.
template <typename T, int V, int HEADS>
__global__ void __launch_bounds__(kThreadsMax) rope_kernel(RopeArgs a)
{
    griddep_wait();
    __shared__ float2 s_cs[kMaxPairs];
    const int64_t t = blockIdx.x;
    const int pairs = a.rope.rotary / 2;
    const int turns = pairs / V, pieces = turns + (a.dim - a.rope.rotary) / V;
    const T *x = static_cast<const T *>(a.x) + t * a.x_st;
    T *y = static_cast<T *>(a.y) + t * a.y_st;
    const int tid = threadIdx.y * blockDim.x + threadIdx.x;
    const int64_t pos = a.rope.positions[t];
    const int h0 = (blockIdx.y * blockDim.y) * HEADS + threadIdx.y;
    bool angles = false;
    for (int p = threadIdx.x; p < pieces || !angles; p += blockDim.x) {
        const bool in = p < pieces, turn = p < turns;
        const int o1 = turn ? (a.rope.interleaved ? 2 * p * V : p * V) : a.rope.rotary + (p - turns) * V;
        const int o2 = a.rope.interleaved ? o1 + V : o1 + pairs;
        Vec<T, V> u[HEADS], w[HEADS];
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {
            const int h = h0 + k * blockDim.y;
            if (in && h < a.heads) {
                u[k] = *reinterpret_cast<const Vec<T, V> *>(x + h * a.x_sh + o1);
                if (turn) w[k] = *reinterpret_cast<const Vec<T, V> *>(x + h * a.x_sh + o2);
            }
        }
        if (!angles) {  // once: the loads above are under way meanwhile
            for (int i = tid; i < pairs; i += blockDim.x * blockDim.y) {
                float2 cs = rope_cos_sin(pos, a.rope.freqs[i], a.rope.scale);
                if (a.rope.backward) cs.y = -cs.y;
                s_cs[i] = cs;
            }
            __syncthreads();
            angles = true;
        }
        if (!in) continue;
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {
            const int h = h0 + k * blockDim.y;
            if (h >= a.heads) continue;
            if (turn) {
                Vec<T, V> r1, r2;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 cs = s_cs[p * V + j];
                    if (a.rope.interleaved) {
                        // elements 2j and 2j + 1 of the 2V read
                        const T x1 = 2 * j < V ? u[k].e[(2 * j) % V] : w[k].e[(2 * j) % V];
                        const T x2 = 2 * j + 1 < V ? u[k].e[(2 * j + 1) % V] : w[k].e[(2 * j + 1) % V];
                        const float2 r = rope_turn(to_f32<T>(x1), to_f32<T>(x2), cs);
                        (2 * j < V ? r1 : r2).e[(2 * j) % V] = from_f32<T>(r.x);
                        (2 * j + 1 < V ? r1 : r2).e[(2 * j + 1) % V] = from_f32<T>(r.y);
                    } else {
                        const float2 r = rope_turn(to_f32<T>(u[k].e[j]), to_f32<T>(w[k].e[j]), cs);
                        r1.e[j] = from_f32<T>(r.x);
                        r2.e[j] = from_f32<T>(r.y);
                    }
                }
                *reinterpret_cast<Vec<T, V> *>(y + h * a.y_sh + o1) = r1;
                *reinterpret_cast<Vec<T, V> *>(y + h * a.y_sh + o2) = r2;
            } else {
                *reinterpret_cast<Vec<T, V> *>(y + h * a.y_sh + o1) = u[k];
            }
        }
    }
}

template <typename T, int V>
cudaError_t launch_v(const RopeArgs &a, int64_t tokens, cudaStream_t s)
{
    const int pieces = a.rope.rotary / 2 / V + (a.dim - a.rope.rotary) / V;
    const int bx = pieces < kThreadsMax ? pieces : kThreadsMax;
    // Four heads per thread keep eight loads in flight and spread the angles
    // over more work; a few tokens are better spread over more threads.
    const bool few = tokens * ((a.heads + 3) / 4) * bx < 152 * 512;
    const int per = few ? 1 : 4;
    int by = (a.heads + per - 1) / per;
    if (by > kThreadsMax / bx) by = kThreadsMax / bx;
    const dim3 grid(static_cast<unsigned>(tokens), static_cast<unsigned>((a.heads + by * per - 1) / (by * per)));
    const dim3 block(bx, by);
    if (few) return launch_pdl(rope_kernel<T, V, 1>, grid, block, 0, s, a);
    return launch_pdl(rope_kernel<T, V, 4>, grid, block, 0, s, a);
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
