// Rotary positions of query and key heads, and the RMS norm of each head in front of them, one pass forward and one backward.
//   z = g x / sqrt(mean(x^2) + eps);   (a, b) -> (a cos - b sin, a sin + b cos)  for the pairs of a head's first `rotated` channels
// The rotation by minus the angle is its transpose: dz = rotation of dy, dg = sum dz xhat, dx = rs (g dz - xhat mean(g dz xhat)).
// HBM bounds both: 8192 positions of 32 / 8 heads of 128 with norms, forward with a second place for x, 77 us, 3.9 TB/s; backward 80 us, 3.8 TB/s;
// 32768 of 16 / 16 heads without norms, 137 us either way, 5.9 TB/s.
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"

namespace bapipe {
namespace {

constexpr int TPB = 256;
constexpr int kGainBlocks = 1024;        // that leave sums of the gains' gradients
constexpr int kMostBlocks = 1 << 22;     // a launch holds less than 2^32 threads; the groups of lanes take what is left in further rounds

template <class T> struct RotaryArgs {
    RotaryShape r;
    const T *x, *dy;
    T *y;                    // or dx
    T *copy;                 // forward: a second place for x, or NULL
    const float2 *table;
    const float *gains;
    float *part;             // [blocks][2][d]
    // forward: query and key heads as 16-bit floats instead, and their scales (AttnArgs); backward: their gradients as floats.  Or NULL
    uint16_t *half;
    float *half_scale;
    const float *dy_float;   // [rows][heads + groups][d]
    int per_row, per_unit;   // heads of a row that are read, and how many of them a group of lanes takes
    int units;
};

template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <int L> __device__ __forceinline__ float group_max(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// A head is taken by L lanes of a wave, a power of two with L V C >= d: C times V neighbouring channels each, C = 1 where V is 16 bytes, which it is
// where d and the turning part (in half layout each half of it) are whole such pieces; else V = 1, C = 8.  A group of L lanes takes K heads
// of a position, all loaded before the first is worked on; their angles are the same.
template <class T, int V, int C, int L, int K, bool PAIRS, bool NORM, bool BACK, bool FLOATS>
__global__ __launch_bounds__(TPB, (BACK && NORM && !FLOATS ? 4 : 1)) void k_rotary(RotaryArgs<T> p)
{
    typedef vec_t<T, V> vec;
    typedef vec_t<float, V> vecf;
    __shared__ float sums[BACK && NORM ? TPB * V * C : 1];
    const RotaryShape &r = p.r;
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = r.d, half = r.rotated / 2;
    const int turning = r.heads + r.groups;
    auto mate_of = [&](int e) { return PAIRS ? e ^ 1 : e < half ? e + half : e - half; };      // of a channel that turns
    float dgain[2][C][V] = {};
    for (int unit = blockIdx.x * (TPB / L) + group; unit < p.units; unit += gridDim.x * (TPB / L)) {
        const int row = unit / p.per_unit, head0 = unit - row * p.per_unit;      // heads head0 + k per_unit
        const float2 *cs = p.table + (size_t)(row % r.T) * half;
        const size_t at_row = (size_t)row * r.stride();
        const T *from = BACK ? p.dy : p.x;
        vec v[K][C], w[K][C], x[K][C];                   // own, the partners' of a half layout, backward the norm's input
        vecf vf[K][C], wf[K][C];                         // FLOATS: instead of the first two
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int head = head0 + k * p.per_unit;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e = (c * L + lane) * V;
                v[k][c] = w[k][c] = x[k][c] = vec{};
                vf[k][c] = wf[k][c] = vecf{};
                if (e >= d || head >= p.per_row) continue;
                const bool turns = head < turning;
                if (FLOATS && turns) {
                    const float *at = p.dy_float + ((size_t)row * turning + head) * d;
                    vf[k][c] = *(const vecf *)(at + e);
                    if (e < r.rotated && (!PAIRS || V == 1)) wf[k][c] = *(const vecf *)(at + mate_of(e));
                } else {
                    const T *at = from + at_row + (size_t)head * d;
                    v[k][c] = *(const vec *)(at + e);
                    if (turns && e < r.rotated && (!PAIRS || V == 1)) w[k][c] = *(const vec *)(at + mate_of(e));
                }
                if (BACK && NORM && turns) x[k][c] = *(const vec *)(p.x + at_row + (size_t)head * d + e);
            }
        }
        float2 angle[C][V];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * L + lane) * V;
            const bool turns = e < r.rotated;
            if (PAIRS) {
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    const float2 a = turns ? cs[(e + j) / 2] : float2{1.0f, 0.0f};
                    angle[c][j] = a;
                    if (V > 1) angle[c][j + (V > 1)] = a;
                }
            } else {
                const float2 *a = cs + (e < half ? e : e - half);
#pragma unroll
                for (int j = 0; j < V; ++j) angle[c][j] = turns ? a[j] : float2{1.0f, 0.0f};
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int head = head0 + k * p.per_unit;
            if (head >= p.per_row) continue;
            const bool turns = head < turning;
            const size_t at = at_row + (size_t)head * d;
            if (!BACK && p.copy) {
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if ((c * L + lane) * V < d) *(vec *)(p.copy + at + (c * L + lane) * V) = v[k][c];
            }
            if (!turns) {
                if (r.values && p.y)
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        if ((c * L + lane) * V < d) *(vec *)(p.y + at + (c * L + lane) * V) = v[k][c];
                continue;
            }
            auto own = [&](int c, int j) { return FLOATS ? vf[k][c].e[j] : to_f32(v[k][c].e[j]); };
            auto mate = [&](int c, int j) {
                if (PAIRS && V > 1) return own(c, j ^ (V > 1 ? 1 : 0));
                return FLOATS ? wf[k][c].e[j] : to_f32(w[k][c].e[j]);
            };
            float rs = 1.0f;
            if (NORM) {
                float squares = 0.0f;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float f = BACK ? to_f32(x[k][c].e[j]) : own(c, j);
                        squares = fmaf(f, f, squares);
                    }
                rs = rsqrtf(group_sum<L>(squares) / d + r.eps);
            }
            const float *gains = NORM ? p.gains + (head < r.heads ? 0 : d) : nullptr;
            float z[C][V], dot = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e0 = (c * L + lane) * V;
                if (e0 >= d) {
#pragma unroll
                    for (int j = 0; j < V; ++j) z[c][j] = 0.0f;
                    continue;
                }
                const bool in = e0 < r.rotated;
                vecf g = {}, gm = {};
                if (NORM) g = *(const vecf *)(gains + e0);
                if (NORM && !BACK && in && (!PAIRS || V == 1)) gm = *(const vecf *)(gains + mate_of(e0));
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float a = own(c, j), b = in ? mate(c, j) : 0.0f;
                    if (NORM && !BACK) {
                        a *= rs * g.e[j];
                        b *= rs * (PAIRS && V > 1 ? g.e[j ^ (V > 1 ? 1 : 0)] : gm.e[j]);
                    }
                    const bool second = PAIRS ? (e0 + j) & 1 : e0 + j >= half;
                    const float sine = second == BACK ? -angle[c][j].y : angle[c][j].y;
                    z[c][j] = fmaf(a, angle[c][j].x, b * sine);
                    if (NORM && BACK) {
                        const float xhat = to_f32(x[k][c].e[j]) * rs;
                        if (head < r.heads) dgain[0][c][j] += z[c][j] * xhat;
                        else dgain[1][c][j] += z[c][j] * xhat;
                        z[c][j] *= g.e[j];
                        dot = fmaf(z[c][j], xhat, dot);
                    }
                }
            }
            if (NORM && BACK) {
                const float mean = group_sum<L>(dot) / d;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < V; ++j) z[c][j] = rs * (z[c][j] - to_f32(x[k][c].e[j]) * rs * mean);
            }
            if (!BACK && p.half) {
                // divided by the power of two that takes the head's largest magnitude to 2^14..2^15 of a format that holds 65504, so that what is
                // 2^28 below it keeps all its digits; infinities and NaN stay what they are
                float most = 0.0f;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < V; ++j) most = fmaxf(most, fabsf(z[c][j]));
                most = group_max<L>(most);
                int up = 0;
                if (most > 0.0f && most < __builtin_inff()) up = min(14 - ilogbf(most), 100);
                if (lane == 0) p.half_scale[(size_t)head * r.rows + row] = ldexpf(1.0f, -up);
                const float by = ldexpf(1.0f, up);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int e = (c * L + lane) * V;
                    if (e >= d) continue;
                    struct alignas(2 * V) {
                        _Float16 e[V];
                    } out;
#pragma unroll
                    for (int j = 0; j < V; ++j) out.e[j] = (_Float16)(z[c][j] * by);
                    __builtin_memcpy(__builtin_assume_aligned(p.half + ((size_t)row * turning + head) * d + e, 2 * V), &out, sizeof out);
                }
                continue;
            }
            if (BACK && !p.y) continue;                  // only the gains want a gradient
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e = (c * L + lane) * V;
                if (e >= d) continue;
                vec out;
#pragma unroll
                for (int j = 0; j < V; ++j) out.e[j] = from_f32<T>(z[c][j]);
                *(vec *)(p.y + at + e) = out;
            }
        }
    }
    if constexpr (BACK && NORM) {
        // the groups of a block, one gain after the other
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) sums[group * (L * C * V) + (c * L + lane) * V + j] = dgain[which][c][j];
            __syncthreads();
            for (int e = threadIdx.x; e < d; e += TPB) {
                float sum = 0.0f;
                for (int g = 0; g < TPB / L; ++g) sum += sums[g * (L * C * V) + e];
                p.part[((size_t)blockIdx.x * 2 + which) * d + e] = sum;
            }
        }
    }
}

// dgains += the blocks' sums; 16 columns and 64 rows to a block
__global__ __launch_bounds__(1024) void k_rotary_gains(const float *part, int blocks, int n, float *dgains)
{
    __shared__ float sums[64][17];
    const int col = threadIdx.x % 16, row = threadIdx.x / 16, e = blockIdx.x * 16 + col;
    float sum = 0.0f;
    if (e < n)
#pragma unroll 8
        for (int b = row; b < blocks; b += 64) sum += part[(size_t)b * n + e];
    sums[row][col] = sum;
    for (int o = 32; o > 0; o /= 2) {
        __syncthreads();
        if (row < o) sums[row][col] += sums[row + o][col];
    }
    if (row == 0 && e < n) dgains[e] += sums[0][col];
}

// Angles in double: a float holds position times frequency to 2^-24 of it, radians at position 10^7
__global__ __launch_bounds__(TPB) void k_rotary_table(float2 *table, size_t n, int half, RotaryAngles a)
{
    const size_t i = (size_t)blockIdx.x * TPB + threadIdx.x;
    if (i >= n) return;
    const int j = (int)(i % half);
    double f = pow(a.base, -(double)j / half);
    if (a.original_length > 0.0) {
        const double turns = a.original_length * f / 6.283185307179586;
        const double kept = fmin(fmax((turns - a.low_turns) / (a.high_turns - a.low_turns), 0.0), 1.0);
        f *= kept + (1.0 - kept) / a.factor;
    } else
        f /= a.factor;
    double sine, cosine;
    sincos((double)(a.first_position + (long long)(i / half)) * f, &sine, &cosine);
    table[i] = {(float)(a.magnitude * cosine), (float)(a.magnitude * sine)};
}

// K: a group of lanes takes two or three heads where there are enough of them for all units of the chip.  More share their angles' loads and
// leave less room for other waves; 8192 positions of 32 / 8 heads of 128 with norms, us forward and backward: one head 98 and -, two 85 and 84,
// three 77 and 80 (3.9 and 3.8 TB/s), four 85 and 93; 32768 of 16 / 16 heads of 128 without: 134, 136, 141, 144 either way; with norms, from float
// gradients, 8192 of 16 / 2 heads: two 38, four 53.
constexpr int rotary_heads(bool norm, bool floats) { return norm && !floats ? 3 : 2; }
constexpr int kManyHeads = 32768;
struct Plan {
    int lanes, K, per_row, per_unit, units, blocks;
    bool vec;
};
Plan plan(int dt, const RotaryShape &r, bool sums, bool all_heads, std::initializer_list<const void *> tensors, int many)
{
    Plan p;
    const int V = 16 / (int)dt_size(dt);
    p.vec = r.d % V == 0 && (r.pairs ? r.rotated % V == 0 : r.rotated / 2 % V == 0);
    for (const void *t : tensors) p.vec = p.vec && (uintptr_t)t % 16 == 0;
    const int pieces = p.vec ? r.d / V : (r.d + 7) / 8;           // without vectors eight channels a lane
    for (p.lanes = 4; p.lanes < pieces;) p.lanes *= 2;
    p.per_row = r.heads + r.groups + (all_heads ? r.groups : 0);
    p.K = p.vec && (long long)r.rows * p.per_row >= kManyHeads ? many : 1;
    p.per_unit = (p.per_row + p.K - 1) / p.K;
    p.units = r.rows * p.per_unit;
    const int per_block = TPB / p.lanes;
    p.blocks = (int)std::min(((long long)p.units + per_block - 1) / per_block, (long long)kMostBlocks);
    if (sums && p.blocks > kGainBlocks) p.blocks = kGainBlocks;
    return p;
}

template <class T, bool NORM, bool BACK, bool FLOATS = false> hipError_t launch(const Plan &p, RotaryArgs<T> a, hipStream_t s)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    a.units = p.units;
    a.per_row = p.per_row;
    a.per_unit = p.per_unit;
#define ROTARY(V, C, L, N)                                                                                                           \
    if (p.vec == (V > 1) && p.lanes == L && p.K == N) {                                                                              \
        if (a.r.pairs) hipLaunchKernelGGL((k_rotary<T, V, C, L, N, true, NORM, BACK, FLOATS>), dim3(p.blocks), dim3(TPB), 0, s, a);  \
        else hipLaunchKernelGGL((k_rotary<T, V, C, L, N, false, NORM, BACK, FLOATS>), dim3(p.blocks), dim3(TPB), 0, s, a);           \
        return hipGetLastError();                                                                                                    \
    }
#define ROTARY_VEC(L) ROTARY(VEC, 1, L, 1) ROTARY(VEC, 1, L, (rotary_heads(NORM, FLOATS)))
    ROTARY_VEC(4) ROTARY_VEC(8) ROTARY_VEC(16) ROTARY_VEC(32)
    if constexpr (VEC == 4) { ROTARY_VEC(64) }
    ROTARY(1, 8, 4, 1) ROTARY(1, 8, 8, 1) ROTARY(1, 8, 16, 1) ROTARY(1, 8, 32, 1)
#undef ROTARY_VEC
#undef ROTARY
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t rotary_table(float2 *table, int T, int rotated, const RotaryAngles &a, hipStream_t s)
{
    const size_t n = (size_t)T * (rotated / 2);
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL(k_rotary_table, dim3((unsigned)((n + TPB - 1) / TPB)), dim3(TPB), 0, s, table, n, rotated / 2, a);
    return hipGetLastError();
}

template <class T>
static hipError_t forward(const RotaryShape &r, const void *x, void *y, const float2 *table, const float *gains, hipStream_t s, void *half, float *half_scale, void *copy)
{
    const Plan p = plan(sizeof(T) == 4 ? DT_F32 : DT_BF16, r, false, r.values || copy, {x, y, half, copy}, rotary_heads(r.eps > 0.0f, false));
    RotaryArgs<T> a = {};
    a.r = r;
    a.x = (const T *)x;
    a.y = (T *)y;
    a.copy = (T *)copy;
    a.table = table;
    a.gains = gains;
    a.half = (uint16_t *)half;
    a.half_scale = half_scale;
    return r.eps > 0.0f ? launch<T, true, false>(p, a, s) : launch<T, false, false>(p, a, s);
}

hipError_t rotary_fwd(int dt, const RotaryShape &r, const void *x, void *y, const float2 *table, const float *gains, hipStream_t s, void *half, float *half_scale,
                      void *copy)
{
    return dt == DT_F32 ? forward<float>(r, x, y, table, gains, s, half, half_scale, copy) : forward<bf16_t>(r, x, y, table, gains, s, half, half_scale, copy);
}

size_t rotary_workspace(int dt, const RotaryShape &r)
{
    // tensors at odd addresses are not read in vectors: a head to a group of no more lanes, so as many blocks or kGainBlocks at most
    if (!(r.eps > 0.0f)) return 0;
    const Plan a = plan(dt, r, true, r.values, {}, 1), b = plan(dt, r, true, r.values, {(const void *)1}, 1);
    return (size_t)(a.blocks > b.blocks ? a.blocks : b.blocks) * 2 * r.d * sizeof(float);
}

template <class T>
static hipError_t backward(const RotaryShape &r, const void *x, const void *dy, const float *dy_float, void *dx, const float2 *table, const float *gains, float *dgains,
                           void *workspace, hipStream_t s)
{
    const bool norm = r.eps > 0.0f;
    if (!norm && !dx) return hipSuccess;
    const Plan p = plan(sizeof(T) == 4 ? DT_F32 : DT_BF16, r, norm, r.values, {x, dy, dx, dy_float}, rotary_heads(norm, dy_float));
    RotaryArgs<T> a = {};
    a.r = r;
    a.x = (const T *)x;
    a.dy = (const T *)dy;
    a.y = (T *)dx;
    a.table = table;
    a.gains = gains;
    a.part = (float *)workspace;
    a.dy_float = dy_float;
    hipError_t e;
    if constexpr (sizeof(T) == 2) {
        if (dy_float) e = norm ? launch<T, true, true, true>(p, a, s) : launch<T, false, true, true>(p, a, s);
        else e = norm ? launch<T, true, true>(p, a, s) : launch<T, false, true>(p, a, s);
    } else
        e = norm ? launch<T, true, true>(p, a, s) : launch<T, false, true>(p, a, s);
    if (e != hipSuccess || !norm) return e;
    hipLaunchKernelGGL(k_rotary_gains, dim3((unsigned)((2 * r.d + 15) / 16)), dim3(1024), 0, s, (const float *)workspace, p.blocks, 2 * r.d, dgains);
    return hipGetLastError();
}

hipError_t rotary_bwd(int dt, const RotaryShape &r, const void *x, const void *dy, const float *dy_float, void *dx, const float2 *table, const float *gains,
                      float *dgains, void *workspace, hipStream_t s)
{
    return dt == DT_F32 ? backward<float>(r, x, dy, dy_float, dx, table, gains, dgains, workspace, s)
                        : backward<bf16_t>(r, x, dy, dy_float, dx, table, gains, dgains, workspace, s);
}

}  // namespace bapipe
