// The norm of each head and rotary positions of one or several axes in one pass,
// for sm_103a, and their gradient:
//   n = x r,  r = (mean x^2 + eps)^-1/2,  y = R (n w)
//   g = R' dy,  dx = r (g w - n mean(g w n)),  dw = sum over tokens and heads of g n
// (R turns pair i by position[axis of i] times frequency i; R' is its transpose),
// and R or R' alone.
//
// HBM-bound: x (and dy) read and y (dx) written once, some 5 to 15 operations per
// element.  A row (a head of a token) belongs to a group of 4 to 32 lanes, each
// with V pairs (two vectors) or V elements that are not turned; the sums over the
// head, in binary32, go across the lanes, and the next row's loads are under way
// meanwhile.  A CTA takes blocks of tokens of one side (queries or keys), whose
// angles it computes once for all their heads: an angle costs about as much as
// six heads' pairs.  dw: each lane sums its elements over its rows, a CTA joins
// its groups, a second kernel the CTAs; all in a fixed order.
#include "quartz_internal.h"
#include "rope.cuh"

namespace quartz {
namespace {

constexpr int kThreads = 256;
constexpr int kMostHere = 16;  // tokens of a block

enum Mode { kRotate, kForward, kBackward };

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

__device__ __forceinline__ float weight_at(const void *w, int type, int i)
{
    if (!w) return 1.f;
    if (type == QUARTZ_OUT_F32) return static_cast<const float *>(w)[i];
    if (type == QUARTZ_OUT_F16) return __half2float(static_cast<const __half *>(w)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[i]);
}

// Elements a lane's piece p holds: pairs p V .. as two vectors (first, first +
// gap), or V elements behind the turned ones (a second vector of nothing).
struct Piece {
    int first, gap;
    bool in, turn;
};

// What a side's CTA sums for dw: [group][element], added up in group order.
// L lanes a row, NP pieces a lane (L NP >= pieces).
template <typename T, int V, int NP, int MODE>
__global__ void __launch_bounds__(kThreads, MODE == kBackward ? 2 : 4) head_norm_kernel(HeadNormArgs a, int lanes_log2, int here)
{
    griddep_wait();
    extern __shared__ __align__(16) float s_dyn[];
    const int pairs = a.rotary / 2, turns = pairs / V, pieces = turns + (a.dim - a.rotary) / V;
    const int L = 1 << lanes_log2, groups = kThreads >> lanes_log2;
    const int width = L * NP * V;  // places of a head, at [j][piece] for each j < V
    // pairs' units and axes; the block's angles [token][j][piece]; the weights of
    // both vectors [j][piece]
    uint64_t *s_unit = reinterpret_cast<uint64_t *>(s_dyn);
    int *s_axis = reinterpret_cast<int *>(s_unit + pairs);
    float2 *s_w = reinterpret_cast<float2 *>(s_axis + ((pairs + 1) & ~1));
    float2 *s_cs = s_w + (MODE == kRotate ? 0 : width);

    const int side = static_cast<int>(blockIdx.x) >= a.ctas[0];
    const int cta = static_cast<int>(blockIdx.x) - (side ? a.ctas[0] : 0), ctas = a.ctas[side];
    const int heads = a.side[side].heads;
    const int group = threadIdx.x >> lanes_log2, lane = threadIdx.x & (L - 1);

    Piece pc[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int p = lane + i * L;
        pc[i].in = p < pieces;
        pc[i].turn = p < turns;
        pc[i].first = !pc[i].in ? 0 : pc[i].turn ? (a.interleaved ? 2 * p * V : p * V) : a.rotary + (p - turns) * V;
        pc[i].gap = a.interleaved ? V : pairs;
    }
    // element of the first (x) and second (y) vector's place j of piece p
    auto element = [&](int p, int j, int second) {
        if (p < turns) return a.interleaved ? 2 * (p * V + j) + second : p * V + j + second * pairs;
        return a.rotary + (p - turns) * V + j;
    };
    for (int i = threadIdx.x; i < pairs; i += kThreads) {
        s_unit[i] = rope_unit(a.freqs[i]);
        int axis = a.pair_axis ? a.pair_axis[i] : 0;
        if (axis < 0 || axis >= a.axes) {
            atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
            axis = 0;
        }
        s_axis[i] = axis;
    }
    if (MODE != kRotate)
        for (int i = threadIdx.x; i < width; i += kThreads) {
            const int j = i / (L * NP), p = i - j * (L * NP);
            float2 w = make_float2(0.f, 0.f);
            if (p < pieces) {
                w.x = weight_at(a.side[side].w, a.w_type, element(p, j, 0));
                if (p < turns) w.y = weight_at(a.side[side].w, a.w_type, element(p, j, 1));
            }
            s_w[i] = w;
        }

    const HeadNormSide &sd = a.side[side];
    const int step_t = groups / heads, step_h = groups - step_t * heads;  // from a group's row to its next
    float dw[MODE == kBackward ? NP : 1][2][MODE == kBackward ? V : 1];
    if (MODE == kBackward)
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) dw[i][0][j] = dw[i][1][j] = 0.f;

    for (int64_t t0 = static_cast<int64_t>(cta) * here; t0 < a.tokens; t0 += static_cast<int64_t>(ctas) * here) {
        const int its = static_cast<int>(min(static_cast<int64_t>(here), a.tokens - t0));
        const int rows = its * heads;
        // the row's vectors; the loads of a row that is not there are left out
        Vec<T, V> u[NP], w[NP], du[MODE == kBackward ? NP : 1], dv[MODE == kBackward ? NP : 1];
        auto load = [&](int t, int h, Vec<T, V>(&u)[NP], Vec<T, V>(&w)[NP], Vec<T, V>(&du)[MODE == kBackward ? NP : 1],
                        Vec<T, V>(&dv)[MODE == kBackward ? NP : 1]) {
            if (t >= its) return;
            const T *x = static_cast<const T *>(sd.x) + (t0 + t) * sd.x_st + h * sd.x_sh;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (pc[i].in) u[i] = *reinterpret_cast<const Vec<T, V> *>(x + pc[i].first);
                if (pc[i].turn) w[i] = *reinterpret_cast<const Vec<T, V> *>(x + pc[i].first + pc[i].gap);
            }
            if constexpr (MODE == kBackward) {
                const T *d = static_cast<const T *>(sd.dy) + (t0 + t) * sd.dy_st + h * sd.dy_sh;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    if (pc[i].in) du[i] = *reinterpret_cast<const Vec<T, V> *>(d + pc[i].first);
                    if (pc[i].turn) dv[i] = *reinterpret_cast<const Vec<T, V> *>(d + pc[i].first + pc[i].gap);
                }
            }
        };
        int t = group / heads, h = group - t * heads;
        load(t, h, u, w, du, dv);  // under way while the angles are computed
        __syncthreads();            // the units; the block before is done with its angles
        for (int i = threadIdx.x; i < its * pairs; i += kThreads) {
            const int k = i / pairs, j = i - k * pairs;
            float2 cs = rope_cos_sin(a.positions[s_axis[j] * a.axis_stride + t0 + k], s_unit[j], a.scale);
            if (MODE == kBackward || (MODE == kRotate && a.backward)) cs.y = -cs.y;
            s_cs[k * width + (j % V) * (L * NP) + j / V] = cs;
        }
        __syncthreads();
        for (int row0 = 0; row0 < rows; row0 += groups) {  // as often for every lane of a warp
            const bool in = t < its;
            int t2 = t + step_t, h2 = h + step_h;
            if (h2 >= heads) h2 -= heads, ++t2;
            Vec<T, V> u2[NP], w2[NP], du2[MODE == kBackward ? NP : 1], dv2[MODE == kBackward ? NP : 1];
            load(t2, h2, u2, w2, du2, dv2);
            const float2 *cs = s_cs + (in ? t : 0) * width + lane;
            const float2 *ws = s_w + lane;
            // places (first, second) of piece i, element j: with `interleaved` a pair's
            // two elements lie side by side over both vectors
            auto x1 = [&](const Vec<T, V> &u, const Vec<T, V> &w, int j, bool turn) {
                if (!a.interleaved || !turn) return to_f32<T>(u.e[j]);
                return to_f32<T>(2 * j < V ? u.e[(2 * j) % V] : w.e[(2 * j) % V]);
            };
            auto x2 = [&](const Vec<T, V> &u, const Vec<T, V> &w, int j) {
                if (!a.interleaved) return to_f32<T>(w.e[j]);
                return to_f32<T>(2 * j + 1 < V ? u.e[(2 * j + 1) % V] : w.e[(2 * j + 1) % V]);
            };
            float r = 1.f, along = 0.f;
            float g[MODE == kBackward ? NP : 1][2][MODE == kBackward ? V : 1];
            if (MODE != kRotate) {
                float ss = 0.f, dot = 0.f;
                if (in) {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        if (!pc[i].in) continue;
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const float a1 = x1(u[i], w[i], j, pc[i].turn), a2 = pc[i].turn ? x2(u[i], w[i], j) : 0.f;
                            ss += a1 * a1;
                            ss += a2 * a2;
                            if constexpr (MODE == kBackward) {
                                const float d1 = x1(du[i], dv[i], j, pc[i].turn);
                                float2 gg = make_float2(d1, 0.f);
                                if (pc[i].turn) gg = rope_turn(d1, x2(du[i], dv[i], j), cs[j * (L * NP) + i * L]);
                                const float2 wt = ws[j * (L * NP) + i * L];
                                g[i][0][j] = gg.x, g[i][1][j] = gg.y;
                                dot += gg.x * wt.x * a1;
                                dot += gg.y * wt.y * a2;
                            }
                        }
                    }
                }
                for (int d = 1; d < L; d *= 2) {
                    ss += __shfl_xor_sync(0xffffffffu, ss, d);
                    if (MODE == kBackward) dot += __shfl_xor_sync(0xffffffffu, dot, d);
                }
                r = rsqrtf(ss * a.inv_dim + a.eps);
                along = r * r * dot * a.inv_dim;
            }
            if (in) {
                T *y = static_cast<T *>(sd.y) + (t0 + t) * sd.y_st + h * sd.y_sh;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    if (!pc[i].in) continue;
                    if (MODE == kRotate && !pc[i].turn) {
                        *reinterpret_cast<Vec<T, V> *>(y + pc[i].first) = u[i];
                        continue;
                    }
                    float f[2][V];  // the two vectors' elements
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float a1 = x1(u[i], w[i], j, pc[i].turn), a2 = pc[i].turn ? x2(u[i], w[i], j) : 0.f;
                        float2 v;
                        if constexpr (MODE == kBackward) {
                            const float2 wt = ws[j * (L * NP) + i * L];
                            v.x = r * (g[i][0][j] * wt.x - a1 * along);
                            v.y = r * (g[i][1][j] * wt.y - a2 * along);
                            dw[i][0][j] += g[i][0][j] * (a1 * r);
                            dw[i][1][j] += g[i][1][j] * (a2 * r);
                        } else {
                            if (MODE == kForward) {
                                const float2 wt = ws[j * (L * NP) + i * L];
                                a1 *= r * wt.x, a2 *= r * wt.y;
                            }
                            v = pc[i].turn ? rope_turn(a1, a2, cs[j * (L * NP) + i * L]) : make_float2(a1, 0.f);
                        }
                        if (a.interleaved && pc[i].turn) {
                            f[2 * j / V][(2 * j) % V] = v.x;
                            f[(2 * j + 1) / V][(2 * j + 1) % V] = v.y;
                        } else {
                            f[0][j] = v.x;
                            f[1][j] = v.y;
                        }
                    }
                    store_rounded<T, V>(y + pc[i].first, f[0]);
                    if (pc[i].turn) store_rounded<T, V>(y + pc[i].first + pc[i].gap, f[1]);
                }
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                u[i] = u2[i], w[i] = w2[i];
                if constexpr (MODE == kBackward) du[i] = du2[i], dv[i] = dv2[i];
            }
            t = t2, h = h2;
        }
    }
    if constexpr (MODE == kBackward) {
        if (!a.part) return;
        // the groups' sums, [group][element], over the angles' memory
        float *s_dw = reinterpret_cast<float *>(s_w);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int p = lane + i * L;
                if (pc[i].in) s_dw[group * a.dim + element(p, j, 0)] = dw[i][0][j];
                if (pc[i].turn) s_dw[group * a.dim + element(p, j, 1)] = dw[i][1][j];
            }
        __syncthreads();
        for (int d = threadIdx.x; d < a.dim; d += kThreads) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g) s += s_dw[g * a.dim + d];
            a.part[static_cast<int64_t>(blockIdx.x) * a.dim + d] = s;
        }
    }
}

// dw of side blockIdx.y, 32 elements per CTA: each warp sums every eighth of the
// side's parts, then the warps are added up.
__global__ void __launch_bounds__(kThreads) head_norm_sum_kernel(HeadNormArgs a)
{
    griddep_wait();
    __shared__ float s_sum[kThreads / 32][32];
    const int side = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = blockIdx.x * 32 + lane;
    if (!a.side[side].dw) return;
    const float *part = a.part + (side ? static_cast<int64_t>(a.ctas[0]) * a.dim : 0) + d;
    float s = 0.f;
    if (d < a.dim) {
#pragma unroll 8
        for (int i = warp; i < a.ctas[side]; i += kThreads / 32) s += part[static_cast<int64_t>(i) * a.dim];
    }
    s_sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && d < a.dim) {
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) s += s_sum[w][lane];
        if (a.w_type == QUARTZ_OUT_F32) static_cast<float *>(a.side[side].dw)[d] = s;
        else if (a.w_type == QUARTZ_OUT_F16) static_cast<__half *>(a.side[side].dw)[d] = __float2half_rn(s);
        else static_cast<__nv_bfloat16 *>(a.side[side].dw)[d] = __float2bfloat16_rn(s);
    }
}

// Lanes of a row, tokens of a block and CTAs of each side.
struct HeadNormPlan {
    int lanes_log2, here, groups;
    int ctas[2];
};

HeadNormPlan head_norm_plan(const int (&heads)[2], int64_t tokens, int pieces, int per_sm)
{
    HeadNormPlan p;
    p.lanes_log2 = 2;
    while (p.lanes_log2 < 5 && (1 << p.lanes_log2) < pieces) ++p.lanes_log2;
    p.groups = kThreads >> p.lanes_log2;
    const int64_t all = static_cast<int64_t>(heads[0]) + heads[1], wave = static_cast<int64_t>(device_sms()) * per_sm;
    // Blocks of at least four rows a group, so that the last round's empty places
    // are few, while the blocks fill the SMs.
    int here = 1;
    while (here < kMostHere && static_cast<int64_t>(here) * heads[0] < 4 * p.groups &&
           (tokens + 2 * here - 1) / (2 * here) * 2 >= wave)
        here *= 2;
    p.here = here;
    const int64_t blocks = (tokens + here - 1) / here;
    for (int i = 0; i < 2; ++i) {
        int64_t n = heads[i] ? (wave * heads[i] + all - 1) / all : 0;
        p.ctas[i] = static_cast<int>(n < blocks ? n : blocks);
    }
    return p;
}

template <typename T>
bool fits(const HeadNormArgs &a, int mode, int v)
{
    const uintptr_t m = v * sizeof(T) - 1;
    if ((a.rotary / 2) % v || (a.dim - a.rotary) % v) return false;
    for (const HeadNormSide &s : a.side) {
        if (!s.heads) continue;
        int64_t strides = s.x_st | s.x_sh | s.y_st | s.y_sh;
        uintptr_t places = reinterpret_cast<uintptr_t>(s.x) | reinterpret_cast<uintptr_t>(s.y);
        if (mode == kBackward) strides |= s.dy_st | s.dy_sh, places |= reinterpret_cast<uintptr_t>(s.dy);
        if (strides % v || (places & m)) return false;
    }
    return true;
}

// The most CTAs: what the parts' workspace is sized by.
constexpr int kBackwardPerSm = 2, kForwardPerSm = 4;

template <typename T, int V, int NP, int MODE>
cudaError_t launch_v(HeadNormArgs &a, cudaStream_t s)
{
    const int pairs = a.rotary / 2, pieces = pairs / V + (a.dim - a.rotary) / V;
    const int heads[2] = {a.side[0].heads, a.side[1].heads};
    const HeadNormPlan p = head_norm_plan(heads, a.tokens, pieces, MODE == kBackward ? kBackwardPerSm : kForwardPerSm);
    a.ctas[0] = p.ctas[0], a.ctas[1] = p.ctas[1];
    const int width = (1 << p.lanes_log2) * NP * V;
    int bytes = pairs * 8 + ((pairs + 1) & ~1) * 4;
    int rest = (p.here + (MODE == kRotate ? 0 : 1)) * width * 8;
    if (MODE == kBackward && rest < p.groups * a.dim * 4) rest = p.groups * a.dim * 4;
    bytes += rest;
    static_assert(NP * V * 32 <= 256, "shared memory stays below 48 KB");
    return launch_pdl(head_norm_kernel<T, V, NP, MODE>, dim3(static_cast<unsigned>(p.ctas[0] + p.ctas[1])), dim3(kThreads), bytes, s, a,
                      p.lanes_log2, p.here);
}

// The widest vectors (16 bytes, or 8) that sizes, strides and addresses allow;
// else one element at a time.  Pieces a lane: for heads of up to 256.
template <typename T, int MODE>
cudaError_t launch_t(HeadNormArgs &a, cudaStream_t s)
{
    constexpr int wide = 16 / sizeof(T), np = sizeof(T) == 4 ? 2 : 1;
    if (fits<T>(a, MODE, wide)) return launch_v<T, wide, np, MODE>(a, s);
    if (fits<T>(a, MODE, wide / 2)) return launch_v<T, wide / 2, 2 * np, MODE>(a, s);
    return launch_v<T, 1, 8, MODE>(a, s);
}

template <int MODE>
cudaError_t launch_mode(HeadNormArgs &a, cudaStream_t s)
{
    if (a.type == QUARTZ_OUT_F16) return launch_t<__half, MODE>(a, s);
    if (a.type == QUARTZ_OUT_BF16) return launch_t<__nv_bfloat16, MODE>(a, s);
    return launch_t<float, MODE>(a, s);
}

}  // namespace

size_t head_norm_workspace_bytes(int dim) { return (static_cast<size_t>(device_sms()) * kBackwardPerSm + 2) * dim * 4; }

cudaError_t launch_rope_axes(HeadNormArgs a, cudaStream_t s) { return launch_mode<kRotate>(a, s); }

cudaError_t launch_head_norm(HeadNormArgs a, cudaStream_t s) { return launch_mode<kForward>(a, s); }

cudaError_t launch_head_norm_backward(HeadNormArgs a, cudaStream_t s)
{
    cudaError_t e = cudaSuccess;
    // sets the CTAs of each side; else both sums are 0
    if (a.tokens > 0 && a.side[0].heads + a.side[1].heads > 0) e = launch_mode<kBackward>(a, s);
    if (e != cudaSuccess || !a.part) return e;
    return launch_pdl(head_norm_sum_kernel, dim3((a.dim + 31) / 32, 2), dim3(kThreads), 0, s, a);
}

}  // namespace quartz
