// Rotary positions of query and key heads, and the RMS norm of each head in front of them, one pass forward and one backward.
//   z = g x / sqrt(mean(x^2) + eps);   (a, b) -> (a cos - b sin, a sin + b cos)  for the pairs of a head's first `rotated` channels
// The rotation by minus the angle is its transpose: dz = rotation of dy, dg = sum dz xhat, dx = rs (g dz - xhat mean(g dz xhat)).
#include "dev_common.h"
#include "kernels.h"

namespace bapipe {
namespace {

constexpr int TPB = 256;
constexpr int kGainBlocks = 1024;        // that leave sums of the gains' gradients

// A head is taken by L lanes of a wave, a power of two, V neighbouring channels each (so L V >= d: one access a lane and tensor).
// V = 16 bytes where every head, and in half layout each half of the turning part, is whole such pieces; else 1, with C channels a lane.
template <class T> struct RotaryArgs {
    RotaryShape r;
    const T *x, *dy;
    T *y;                    // or dx
    const float2 *table;
    const float *gains;
    float *part;             // [blocks][2][d]
    // forward: query and key heads once more as 16-bit floats, and their scales (AttnArgs); backward: their gradients as floats.  Or NULL
    uint16_t *half;
    float *half_scale;
    const float *dy_float;   // [rows][heads + groups][d]
    int units;               // heads of all positions
};

// turned value at channel e of its head from its own and its partner's value; sign: -1 turns back
template <bool PAIRS> __device__ __forceinline__ int partner(int e, int rotated)
{
    if (PAIRS) return e ^ 1;
    return e < rotated / 2 ? e + rotated / 2 : e - rotated / 2;
}
template <bool PAIRS> __device__ __forceinline__ float turn(float own, float other, float2 cs, bool second, float sign)
{
    return fmaf(own, cs.x, (second ? sign : -sign) * other * cs.y);
}

template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// V channels a lane, C accesses of them, L lanes to a head
template <class T, int V, int C, int L, bool PAIRS, bool NORM, bool BACK, bool FLOATS>
__global__ __launch_bounds__(TPB) void k_rotary(RotaryArgs<T> p)
{
    typedef vec_t<T, V> vec;
    typedef vec_t<float, V> vecf;
    __shared__ float sums[BACK && NORM ? TPB * V * C : 1];
    const RotaryShape &r = p.r;
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = r.d, half = r.rotated / 2;
    const int turning = r.heads + r.groups, per_row = turning + (r.values ? r.groups : 0);
    float dgain[2][C][V] = {};
    for (int unit = blockIdx.x * (TPB / L) + group; unit < p.units; unit += gridDim.x * (TPB / L)) {
        const int row = unit / per_row, head = unit - row * per_row;
        const size_t at = (size_t)row * r.stride() + (size_t)head * d;
        const bool turns = head < turning;
        const float2 *cs = p.table + (size_t)(row % r.T) * half;
        const T *from = BACK ? p.dy : p.x;
        float v[C][V], w[C][V];                          // own, the partners' of a half layout
        vec x[C];                                        // backward the norm's input
        auto load = [&](float (&to)[V], int e) {
            if (FLOATS && turns) {
                const vecf f = *(const vecf *)(p.dy_float + ((size_t)row * turning + head) * d + e);
#pragma unroll
                for (int j = 0; j < V; ++j) to[j] = f.e[j];
            } else {
                const vec f = *(const vec *)(from + at + e);
#pragma unroll
                for (int j = 0; j < V; ++j) to[j] = to_f32(f.e[j]);
            }
        };
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * L + lane) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) v[c][j] = w[c][j] = 0.0f;
            x[c] = vec{};
            if (e >= d) continue;
            load(v[c], e);
            if (turns && e < r.rotated) {
                if (!PAIRS) load(w[c], partner<false>(e, r.rotated));
                else if (V == 1) load(w[c], e ^ 1);
            }
            if (BACK && NORM && turns) x[c] = *(const vec *)(p.x + at + e);
        }
        float rs = 1.0f;
        if (NORM && turns) {
            float squares = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float f = BACK ? to_f32(x[c].e[j]) : v[c][j];
                    squares = fmaf(f, f, squares);
                }
            rs = rsqrtf(group_sum<L>(squares) / d + r.eps);
        }
        const float *gains = NORM && turns ? p.gains + (head < r.heads ? 0 : d) : nullptr;
        float z[C][V], dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e0 = (c * L + lane) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int e = e0 + j;
                float own = v[c][j];
                if (!turns || e >= d) { z[c][j] = own; continue; }
                float other = 0.0f;
                float2 angle = {1.0f, 0.0f};
                bool second = false;
                const int mate = partner<PAIRS>(e, r.rotated);
                if (e < r.rotated) {
                    other = PAIRS && V > 1 ? v[c][j ^ (V > 1 ? 1 : 0)] : w[c][j];
                    angle = cs[PAIRS ? e >> 1 : e < half ? e : e - half];
                    second = PAIRS ? e & 1 : e >= half;
                }
                if (NORM && !BACK) {
                    own *= rs * gains[e];
                    if (e < r.rotated) other *= rs * gains[mate];
                }
                z[c][j] = turn<PAIRS>(own, other, angle, second, BACK ? -1.0f : 1.0f);
                if (NORM && BACK) {
                    const float xhat = to_f32(x[c].e[j]) * rs;
                    if (head < r.heads) dgain[0][c][j] += z[c][j] * xhat;
                    else dgain[1][c][j] += z[c][j] * xhat;
                    z[c][j] *= gains[e];
                    dot = fmaf(z[c][j], xhat, dot);
                }
            }
        }
        if (NORM && BACK && turns) {
            const float mean = group_sum<L>(dot) / d;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) z[c][j] = rs * (z[c][j] - to_f32(x[c].e[j]) * rs * mean);
        }
        if (BACK && !p.y) continue;                      // only the gains want a gradient
        if (!BACK && p.half && turns) {
            // divided by the power of two that takes the head's largest magnitude to 2^14..2^15 of a format that holds 65504, so that what is
            // 2^28 below it keeps all its digits; infinities and NaN stay what they are
            float most = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if ((c * L + lane) * V + j < d) most = fmaxf(most, fabsf(z[c][j]));
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
            int up = 0;
            if (most > 0.0f && most < __builtin_inff()) up = min(14 - ilogbf(most), 100);
            if (lane == 0) p.half_scale[(size_t)head * r.rows + row] = ldexpf(1.0f, -up);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e = (c * L + lane) * V;
                if (e >= d) continue;
                struct alignas(2 * V) {
                    _Float16 e[V];
                } out;
#pragma unroll
                for (int j = 0; j < V; ++j) out.e[j] = (_Float16)ldexpf(z[c][j], up);
                __builtin_memcpy(__builtin_assume_aligned(p.half + ((size_t)row * turning + head) * d + e, 2 * V), &out, sizeof out);
            }
        }
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

// dgains += the blocks' sums; 16 columns and 16 rows to a block
__global__ __launch_bounds__(TPB) void k_rotary_gains(const float *part, int blocks, int n, float *dgains)
{
    __shared__ float sums[16][17];
    const int col = threadIdx.x % 16, row = threadIdx.x / 16, e = blockIdx.x * 16 + col;
    float sum = 0.0f;
    for (int b = row; b < blocks && e < n; b += 16) sum += part[(size_t)b * n + e];
    sums[row][col] = sum;
    __syncthreads();
    if (row == 0 && e < n) {
        sum = 0.0f;
        for (int i = 0; i < 16; ++i) sum += sums[i][col];
        dgains[e] += sum;
    }
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

struct Plan {
    int lanes, units, blocks;
    bool vec;
};
Plan plan(int dt, const RotaryShape &r, bool sums, std::initializer_list<const void *> tensors)
{
    Plan p;
    const int V = 16 / (int)dt_size(dt);
    p.vec = r.d % V == 0 && (r.pairs || r.rotated / 2 % V == 0);
    for (const void *t : tensors) p.vec = p.vec && (uintptr_t)t % 16 == 0;
    const int pieces = p.vec ? r.d / V : (r.d + 7) / 8;           // without vectors eight channels a lane
    for (p.lanes = 4; p.lanes < pieces;) p.lanes *= 2;
    p.units = r.rows * (r.heads + r.groups + (r.values ? r.groups : 0));
    const int per_block = TPB / p.lanes;
    p.blocks = (int)(((long long)p.units + per_block - 1) / per_block);
    if (sums && p.blocks > kGainBlocks) p.blocks = kGainBlocks;
    return p;
}

template <class T, bool NORM, bool BACK, bool FLOATS = false> hipError_t launch(const Plan &p, RotaryArgs<T> a, hipStream_t s)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    a.units = p.units;
#define ROTARY(V, C, L)                                                                                                          \
    if (p.vec == (V > 1) && p.lanes == L) {                                                                                      \
        if (a.r.pairs) hipLaunchKernelGGL((k_rotary<T, V, C, L, true, NORM, BACK, FLOATS>), dim3(p.blocks), dim3(TPB), 0, s, a); \
        else hipLaunchKernelGGL((k_rotary<T, V, C, L, false, NORM, BACK, FLOATS>), dim3(p.blocks), dim3(TPB), 0, s, a);          \
        return hipGetLastError();                                                                                                \
    }
    ROTARY(VEC, 1, 4) ROTARY(VEC, 1, 8) ROTARY(VEC, 1, 16) ROTARY(VEC, 1, 32)
    if constexpr (VEC == 4) { ROTARY(VEC, 1, 64) }
    ROTARY(1, 8, 4) ROTARY(1, 8, 8) ROTARY(1, 8, 16) ROTARY(1, 8, 32)
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

hipError_t rotary_fwd(int dt, const RotaryShape &r, const void *x, void *y, const float2 *table, const float *gains, hipStream_t s, void *half, float *half_scale)
{
    const Plan p = plan(dt, r, false, {x, y, half});
    const bool norm = r.eps > 0.0f;
    if (dt == DT_F32) {
        const RotaryArgs<float> a{r, (const float *)x, nullptr, (float *)y, table, gains, nullptr, nullptr, nullptr, nullptr, 0};
        return norm ? launch<float, true, false>(p, a, s) : launch<float, false, false>(p, a, s);
    }
    const RotaryArgs<bf16_t> a{r, (const bf16_t *)x, nullptr, (bf16_t *)y, table, gains, nullptr, (uint16_t *)half, half_scale, nullptr, 0};
    return norm ? launch<bf16_t, true, false>(p, a, s) : launch<bf16_t, false, false>(p, a, s);
}

size_t rotary_workspace(int dt, const RotaryShape &r)
{
    // tensors at odd addresses are not read in vectors: no more lanes to a head, so no more blocks
    return r.eps > 0.0f ? (size_t)plan(dt, r, true, {}).blocks * 2 * r.d * sizeof(float) : 0;
}

hipError_t rotary_bwd(int dt, const RotaryShape &r, const void *x, const void *dy, const float *dy_float, void *dx, const float2 *table, const float *gains,
                      float *dgains, void *workspace, hipStream_t s)
{
    const bool norm = r.eps > 0.0f;
    if (!norm && !dx) return hipSuccess;
    const Plan p = plan(dt, r, norm, {x, dy, dx, dy_float});
    float *part = (float *)workspace;
    hipError_t e;
    if (dt == DT_F32) {
        const RotaryArgs<float> a{r, (const float *)x, (const float *)dy, (float *)dx, table, gains, part, nullptr, nullptr, nullptr, 0};
        e = norm ? launch<float, true, true>(p, a, s) : launch<float, false, true>(p, a, s);
    } else {
        const RotaryArgs<bf16_t> a{r, (const bf16_t *)x, (const bf16_t *)dy, (bf16_t *)dx, table, gains, part, nullptr, nullptr, dy_float, 0};
        if (dy_float) e = norm ? launch<bf16_t, true, true, true>(p, a, s) : launch<bf16_t, false, true, true>(p, a, s);
        else e = norm ? launch<bf16_t, true, true>(p, a, s) : launch<bf16_t, false, true>(p, a, s);
    }
    if (e != hipSuccess || !norm) return e;
    hipLaunchKernelGGL(k_rotary_gains, dim3((unsigned)((2 * r.d + 15) / 16)), dim3(TPB), 0, s, part, p.blocks, 2 * r.d, dgains);
    return hipGetLastError();
}

}  // namespace bapipe
