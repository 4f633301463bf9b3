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
// head, in binary32, go across the lanes, and the next rows are on their way into
// shared memory meanwhile.  A CTA takes blocks of tokens of one side (queries or
// keys), whose angles it computes once for all their heads: an angle costs about as
// much as three heads' pairs.  dw: each lane sums its elements over its rows, a CTA
// joins its groups, a second kernel the CTAs; all in a fixed order.
// Measured (bf16; us, of the copy rate): gradient of 8192 x 40 heads of 128 73, 50%
// (230 with angles and weights from shared memory for each row, 170 in registers,
// 93 with rows on their way, 73 with instances for lanes full of pairs; then issue
// slots are 64% busy, the rest waits for chains at 4 warps a scheduler); rotation of
// 17550 x 16 heads by three axes 24.1, 88%; fp16, 4608 x 48 heads, forward 28.5, 59%
// (30.5 with three CTAs per SM and rows six ahead).
#pragma once

#include "ptx.cuh"
#include "rope.cuh"

namespace quartz {

constexpr int kNormThreads = 256;
constexpr int kMostHere = 16;  // tokens of a block

enum NormMode { kRotate, kForward, kBackward };

// CTAs per SM: as many as the registers of a lane's vectors, angles, weights and
// sums allow.  16-bit types forward: four where every lane has pairs alone (4608 x
// 48 heads of 128: 28.5 us, three 30.5), else three, whose code needs the registers
// (8192 x 40 heads of 80: 37 us, four 40.5; 4608 x 48 of 128, element by element:
// 136, 150).
template <typename T, int MODE, int E, bool FULL>  // E: pairs a lane
constexpr int kPerSm = MODE == kRotate ? 4 : MODE == kForward ? (sizeof(T) == 4 ? 2 : FULL ? 4 : 3) : (sizeof(T) * E <= 16 ? 2 : 1);
constexpr int kMostBackward = 2;

// Rows that a lane's copies are ahead, each in memory of its own, so that some
// 128 KB per SM are on their way; elements one at a time are loaded as needed.
template <typename T, int MODE, int V, bool FULL>
constexpr int kAhead = sizeof(T) * V < 8 ? 0 : MODE == kBackward ? 4 : MODE == kForward ? (sizeof(T) == 2 && FULL ? 4 : 6) : 5;

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

// The elements of a vector in binary32.
template <typename T, int V>
__device__ __forceinline__ void to_floats(const Vec<T, V> &v, float (&f)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = to_f32<T>(v.e[j]);
}
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
struct NormPiece {
    int first;
    bool in, turn;
};

// L lanes a row, NP pieces a lane (L NP >= pieces).  A group of L lanes takes one
// token of the block and every (groups / here)-th of its heads, so that a lane's
// angles, as its weights, are in registers.  INTER: pairs lie side by side.  FULL:
// every lane has pairs alone (else a third more instructions, for what is not).
template <typename T, int V, int NP, int MODE, bool INTER, bool FULL>
__global__ void __launch_bounds__(kNormThreads, kPerSm<T, MODE, V * NP, FULL>) head_norm_kernel(HeadNormArgs a, int lanes_log2, int q_here, int k_here)
{
    griddep_wait();
    extern __shared__ __align__(16) float s_dyn[];
    constexpr bool kBack = MODE == kBackward;
    const int pairs = a.rotary / 2, turns = pairs / V, pieces = turns + (a.dim - a.rotary) / V;
    const int L = 1 << lanes_log2, groups = kNormThreads >> lanes_log2;
    const int width = L * NP * V;  // places of a head, at [j][piece] for each j < V
    // pairs' units and axes; the block's angles [token][j][piece]
    uint64_t *s_unit = reinterpret_cast<uint64_t *>(s_dyn);
    int *s_axis = reinterpret_cast<int *>(s_unit + pairs);
    float2 *s_cs = reinterpret_cast<float2 *>(s_axis + ((pairs + 1) & ~1));

    const int side = static_cast<int>(blockIdx.x) >= a.ctas[0];
    const int cta = static_cast<int>(blockIdx.x) - (side ? a.ctas[0] : 0), ctas = a.ctas[side];
    const HeadNormSide &sd = a.side[side];
    const int heads = sd.heads, here = side ? k_here : q_here;
    const int group = threadIdx.x >> lanes_log2, lane = threadIdx.x & (L - 1);
    const int tk = group & (here - 1), sub = group / here, step = groups / here;  // `here` is a power of two

    // pairs side by side in memory, or (V = 1 either way) `gap` apart
    const bool beside = INTER || (V == 1 && a.interleaved);
    NormPiece pc[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int p = lane + i * L;
        pc[i].in = FULL || p < pieces;
        pc[i].turn = FULL || p < turns;
        pc[i].first = !pc[i].in ? 0 : pc[i].turn ? (beside ? 2 * p * V : p * V) : a.rotary + (p - turns) * V;
    }
    const int gap = beside ? V : pairs;
    // element of the first (x) and second (y) of a pair, place j of piece p
    auto element = [&](int p, int j, int second) {
        if (FULL || p < turns) return beside ? 2 * (p * V + j) + second : p * V + j + second * pairs;
        return a.rotary + (p - turns) * V + j;
    };
    for (int i = threadIdx.x; i < pairs; i += kNormThreads) {
        s_unit[i] = rope_unit(a.freqs[i]);
        int axis = a.pair_axis ? a.pair_axis[i] : 0;
        if (axis < 0 || axis >= a.axes) {
            atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
            axis = 0;
        }
        s_axis[i] = axis;
    }
    constexpr int NW = MODE == kRotate ? 1 : NP, VW = MODE == kRotate ? 1 : V, ND = kBack ? NP : 1, VD = kBack ? V : 1;
    float w1[NW][VW], w2[NW][VW], dw1[ND][VD], dw2[ND][VD];
    if (MODE != kRotate)
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                w1[i][j] = pc[i].in ? weight_at(sd.w, a.w_type, element(lane + i * L, j, 0)) : 0.f;
                w2[i][j] = pc[i].turn ? weight_at(sd.w, a.w_type, element(lane + i * L, j, 1)) : 0.f;
            }
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < VD; ++j) dw1[i][j] = dw2[i][j] = 0.f;

    // The pairs of two vectors; a piece that is not turned has zeros for its seconds,
    // one that is not there zeros.  (Of a row that is not there they may be anything.)
    auto pairs_of = [&](const Vec<T, V> &u, const Vec<T, V> &v, bool in, bool turn, float (&x1)[V], float (&x2)[V]) {
        float f[2][V];
        to_floats<T, V>(u, f[0]);
        to_floats<T, V>(v, f[1]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (INTER && turn) x1[j] = f[2 * j / V][2 * j % V], x2[j] = f[(2 * j + 1) / V][(2 * j + 1) % V];
            else x1[j] = f[0][j], x2[j] = f[1][j];
        }
        if (!turn)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x2[j] = 0.f;
                if (!in) x1[j] = 0.f;
            }
    };
    // The rows' vectors on their way: [stage][vector][thread], read by the lane that
    // copies them alone.  `ahead` is the row that is asked for next.
    constexpr int S = kAhead<T, MODE, V, FULL>, kVecs = (kBack ? 4 : 2) * NP;
    Vec<T, V> *s_ring = reinterpret_cast<Vec<T, V> *>(reinterpret_cast<uint8_t *>(s_dyn) + a.ring_at) + threadIdx.x;
    const int rounds = (heads + step - 1) / step;  // as often for every lane of a warp
    const int64_t stride = static_cast<int64_t>(ctas) * here;
    int64_t t_ahead = static_cast<int64_t>(cta) * here;  // of a block
    int n_ahead = 0, stage_ahead = 0, stage = 0;
    auto vectors = [&](int64_t t, int h, auto take) {
        const T *from = static_cast<const T *>(sd.x) + t * sd.x_st + h * sd.x_sh;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (pc[i].in) take(2 * i, from + pc[i].first);
            if (pc[i].turn) take(2 * i + 1, from + pc[i].first + gap);
        }
        if constexpr (kBack) {
            const T *d = static_cast<const T *>(sd.dy) + t * sd.dy_st + h * sd.dy_sh;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (pc[i].in) take(2 * NP + 2 * i, d + pc[i].first);
                if (pc[i].turn) take(2 * NP + 2 * i + 1, d + pc[i].first + gap);
            }
        }
    };
    auto ask = [&] {
        if constexpr (S > 0) {
            if (t_ahead + tk < a.tokens && sub + n_ahead * step < heads)
                vectors(t_ahead + tk, sub + n_ahead * step, [&](int k, const T *from) {
                    const uint32_t to = smem_u32(s_ring + (stage_ahead * kVecs + k) * kNormThreads);
                    if constexpr (sizeof(T) * V == 16) cp_async16(to, from);
                    else cp_async8(to, from);
                });
            cp_async_commit();
            stage_ahead = stage_ahead + 1 == S ? 0 : stage_ahead + 1;
            if (++n_ahead == rounds) n_ahead = 0, t_ahead += stride;
        }
    };
    for (int i = 0; i < S - 1; ++i) ask();
    for (int64_t t0 = static_cast<int64_t>(cta) * here; t0 < a.tokens; t0 += stride) {
        const int its = static_cast<int>(min(static_cast<int64_t>(here), a.tokens - t0));
        const int64_t t = t0 + tk;
        const int end = tk < its ? heads : 0;
        T *y = static_cast<T *>(sd.y) + t * sd.y_st;
        __syncthreads();  // the units; the block before is done with its angles
        for (int i = threadIdx.x; i < its * pairs; i += kNormThreads) {
            const int k = i / pairs, j = i - k * pairs;
            float2 cs = rope_cos_sin(a.positions[s_axis[j] * a.axis_stride + t0 + k], s_unit[j], a.scale);
            if (kBack || (MODE == kRotate && a.backward)) cs.y = -cs.y;
            s_cs[k * width + (j % V) * (L * NP) + j / V] = cs;
        }
        __syncthreads();
        float2 cs[NP][V];
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                cs[i][j] = s_cs[tk * width + lane + j * (L * NP) + i * L];
                if (!pc[i].turn) cs[i][j] = make_float2(1.f, 0.f);
            }
        for (int n = 0, h = sub; n < rounds; ++n, h += step) {
            const bool in = h < end;
            Vec<T, V> raw[kVecs];
            ask();
            if constexpr (S > 0) {
                cp_async_wait<S - 1>();
#pragma unroll
                    for (int k = 0; k < kVecs; ++k) raw[k] = s_ring[(stage * kVecs + k) * kNormThreads];
                stage = stage + 1 == S ? 0 : stage + 1;
            } else if (in) {
                vectors(t, h, [&](int k, const T *from) { raw[k] = *reinterpret_cast<const Vec<T, V> *>(from); });
            }
            float x1[NP][V], x2[NP][V], g1[ND][VD], g2[ND][VD], gw1[ND][VD], gw2[ND][VD];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                pairs_of(raw[2 * i], raw[2 * i + 1], pc[i].in, pc[i].turn, x1[i], x2[i]);
                if constexpr (kBack) {
                    pairs_of(raw[2 * NP + 2 * i], raw[2 * NP + 2 * i + 1], pc[i].in, pc[i].turn, g1[i], g2[i]);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float2 g = rope_turn(g1[i][j], g2[i][j], cs[i][j]);
                        g1[i][j] = g.x, g2[i][j] = g.y;
                    }
                }
            }
            float r = 1.f, along = 0.f;  // mean(g w n)
            if (MODE != kRotate) {
                float ss = 0.f, dot = 0.f;
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        ss += x1[i][j] * x1[i][j];
                        ss += x2[i][j] * x2[i][j];
                        if constexpr (kBack) {
                            gw1[i][j] = g1[i][j] * w1[i][j], gw2[i][j] = g2[i][j] * w2[i][j];
                            dot += gw1[i][j] * x1[i][j];
                            dot += gw2[i][j] * x2[i][j];
                        }
                    }
                for (int d = 1; d < L; d *= 2) {
                    ss += __shfl_xor_sync(0xffffffffu, ss, d);
                    if (kBack) dot += __shfl_xor_sync(0xffffffffu, dot, d);
                }
                r = rsqrtf(ss * a.inv_dim + a.eps);
                along = r * dot * a.inv_dim;
            }
            if (!in) continue;
            T *to = y + h * sd.y_sh;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (!pc[i].in) continue;
                float f[2][V];  // the two vectors' elements
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float2 z;
                    if constexpr (kBack) {
                        // by n = x r, not by powers of r, which leave binary32 before x^2 does
                        const float n1 = x1[i][j] * r, n2 = x2[i][j] * r;
                        z.x = r * (gw1[i][j] - n1 * along);
                        z.y = r * (gw2[i][j] - n2 * along);
                        dw1[i][j] += g1[i][j] * n1;
                        dw2[i][j] += g2[i][j] * n2;
                    } else if constexpr (MODE == kForward) {
                        z = rope_turn(x1[i][j] * (r * w1[i][j]), x2[i][j] * (r * w2[i][j]), cs[i][j]);
                    } else {
                        z = rope_turn(x1[i][j], x2[i][j], cs[i][j]);
                    }
                    if (INTER && pc[i].turn) f[2 * j / V][2 * j % V] = z.x, f[(2 * j + 1) / V][(2 * j + 1) % V] = z.y;
                    else f[0][j] = z.x, f[1][j] = z.y;
                }
                store_rounded<T, V>(to + pc[i].first, f[0]);
                if (pc[i].turn) store_rounded<T, V>(to + pc[i].first + gap, f[1]);
            }
        }
    }
    if constexpr (kBack) {
        cp_async_wait<0>();
        if (!a.part) return;
        // the groups' sums, [group][element], over the angles' memory
        float *s_dw = reinterpret_cast<float *>(s_cs);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int p = lane + i * L;
                if (pc[i].in) s_dw[group * a.dim + element(p, j, 0)] = dw1[i][j];
                if (pc[i].turn) s_dw[group * a.dim + element(p, j, 1)] = dw2[i][j];
            }
        __syncthreads();
        for (int d = threadIdx.x; d < a.dim; d += kNormThreads) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g) s += s_dw[g * a.dim + d];
            a.part[static_cast<int64_t>(blockIdx.x) * a.dim + d] = s;
        }
    }
}

// Lanes of a row; tokens of a block and CTAs of each side.
struct HeadNormPlan {
    int lanes_log2, groups;
    int here[2], ctas[2];
};

inline HeadNormPlan head_norm_plan(const int (&heads)[2], int64_t tokens, int pieces, int pairs, int per_sm)
{
    HeadNormPlan p;
    p.lanes_log2 = 2;
    while (p.lanes_log2 < 5 && (1 << p.lanes_log2) < pieces) ++p.lanes_log2;
    p.groups = kNormThreads >> p.lanes_log2;
    const int64_t wave = static_cast<int64_t>(device_sms()) * per_sm;
    // A side's work: its heads, and the angles, which cost about as much as 3.
    const int64_t work[2] = {heads[0] ? heads[0] + 3 : 0, heads[1] ? heads[1] + 3 : 0}, sum = work[0] + work[1];
    for (int i = 0; i < 2; ++i) {
        p.here[i] = 1, p.ctas[i] = 0;
        if (!heads[i]) continue;
        const int64_t most = (wave * work[i] + sum - 1) / sum;
        // Of blocks of 1, 2, .. 16 tokens (one for each group at most) those whose last
        // CTA is done first: in rows a group, a block costs its rows, one for the waits
        // and a third for each angle a thread has.
        int64_t least = 0;
        for (int here = 1; here <= kMostHere && here <= p.groups; here *= 2) {
            const int64_t blocks = (tokens + here - 1) / here, step = p.groups / here;
            const int64_t turns = blocks < most ? 1 : (blocks + most - 1) / most;
            const int64_t cost = turns * (3 * ((heads[i] + step - 1) / step) + 3 + (here * pairs + kNormThreads - 1) / kNormThreads);
            if (here > 1 && cost >= least) continue;
            least = cost;
            p.here[i] = here;
            p.ctas[i] = static_cast<int>(blocks < most ? blocks : most);
        }
    }
    return p;
}

template <typename T>
bool norm_fits(const HeadNormArgs &a, int mode, int v)
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

template <typename T, int V, int NP, int MODE, bool INTER, bool FULL>
cudaError_t launch_norm_v(HeadNormArgs &a, cudaStream_t s)
{
    const int pairs = a.rotary / 2, pieces = pairs / V + (a.dim - a.rotary) / V;
    const int heads[2] = {a.side[0].heads, a.side[1].heads};
    const HeadNormPlan p = head_norm_plan(heads, a.tokens, pieces, pairs, kPerSm<T, MODE, V * NP, FULL>);
    a.ctas[0] = p.ctas[0], a.ctas[1] = p.ctas[1];
    const int width = (1 << p.lanes_log2) * NP * V;
    int bytes = pairs * 8 + ((pairs + 1) & ~1) * 4;
    int rest = (p.here[0] > p.here[1] ? p.here[0] : p.here[1]) * width * 8;
    if (MODE == kBackward && rest < p.groups * a.dim * 4) rest = p.groups * a.dim * 4;
    bytes = (bytes + rest + 15) & ~15;
    static_assert(NP * V * 32 <= 256, "units, angles and sums stay below 37 KB");
    constexpr int kRing = kAhead<T, MODE, V, FULL> * (MODE == kBackward ? 4 : 2) * NP * static_cast<int>(sizeof(T)) * V * kNormThreads;
    a.ring_at = bytes;
    bytes += kRing;
    const cudaError_t e = allow_shared<head_norm_kernel<T, V, NP, MODE, INTER, FULL>>(kRing + 37 * 1024);
    if (e != cudaSuccess) return e;
    return launch_pdl(head_norm_kernel<T, V, NP, MODE, INTER, FULL>, dim3(static_cast<unsigned>(p.ctas[0] + p.ctas[1])), dim3(kNormThreads),
                      bytes, s, a, p.lanes_log2, p.here[0], p.here[1]);
}

// Pieces a lane: one where 32 lanes' are enough (heads of up to 256 elements).
template <typename T, int V, int MODE, bool INTER>
cudaError_t launch_norm_np(HeadNormArgs &a, cudaStream_t s)
{
    const int turns = a.rotary / 2 / V, pieces = turns + (a.dim - a.rotary) / V;
    if constexpr (V * 32 < 256)
        if (pieces > 32) return launch_norm_v<T, V, 256 / V / 32, MODE, INTER, false>(a, s);
    if constexpr (V * sizeof(T) == 16)
        if (pieces == turns && (pieces == 4 || pieces == 8 || pieces == 16 || pieces == 32)) return launch_norm_v<T, V, 1, MODE, INTER, true>(a, s);
    return launch_norm_v<T, V, 1, MODE, INTER, false>(a, s);
}

// The widest vectors (16 bytes, or 8) that sizes, strides and addresses allow;
// else one element at a time.
template <typename T, int MODE>
cudaError_t launch_norm_t(HeadNormArgs &a, cudaStream_t s)
{
    constexpr int wide = 16 / sizeof(T);
    for (int v = wide; v > 1; v /= 2) {
        if (!norm_fits<T>(a, MODE, v)) continue;
        if (v == wide) return a.interleaved ? launch_norm_np<T, wide, MODE, true>(a, s) : launch_norm_np<T, wide, MODE, false>(a, s);
        if (v == wide / 2) return a.interleaved ? launch_norm_np<T, wide / 2, MODE, true>(a, s) : launch_norm_np<T, wide / 2, MODE, false>(a, s);
        break;
    }
    return launch_norm_v<T, 1, 8, MODE, false, false>(a, s);
}

template <int MODE>
cudaError_t launch_norm_mode(HeadNormArgs &a, cudaStream_t s)
{
    if (a.type == QUARTZ_OUT_F16) return launch_norm_t<__half, MODE>(a, s);
    if (a.type == QUARTZ_OUT_BF16) return launch_norm_t<__nv_bfloat16, MODE>(a, s);
    return launch_norm_t<float, MODE>(a, s);
}

// A unit each (head_norm_rotate.cu, head_norm.cu, head_norm_backward.cu); the
// last sets a.ctas.
cudaError_t launch_norm_rotate(HeadNormArgs &a, cudaStream_t s);
cudaError_t launch_norm_forward(HeadNormArgs &a, cudaStream_t s);
cudaError_t launch_norm_backward(HeadNormArgs &a, cudaStream_t s);

}  // namespace quartz
