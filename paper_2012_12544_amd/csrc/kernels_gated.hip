// Gated linear layer, at every position (row) of an NHWC tensor:
//   [g | u] = x W^T + b, W [2F][C] with the F gate rows first;  h = act(g) u
//   D = [dh u act'(g) | dh act(g)];  dx = D W;  dW += D^T x;  db += sum over rows of D
// g and u are kept in float for the backward pass, P [rows][2F].  Rounded to bf16 they were, with D's own rounding, what a
// bf16 layer's gradients were off by most: 3.0e-3 of dW and dx against 64 bits (2-norm), 2.3e-3 so.
// Products of bf16 whose widths are multiples of 8 run on the bf16 matrix cores, the others on the float ones.
#include "dev_common.h"
#include "kernels.h"

namespace bapipe {
namespace {

constexpr int TPB = 256;
typedef float f32x16 __attribute__((ext_vector_type(16)));

// act(g) and its derivative.  A ReLU's derivative at 0 is 0, as everywhere in the library.
__device__ __forceinline__ float act_value(int act, float g)
{
    if (act == ACT_RELU) return fmaxf(g, 0.0f);
    if (act == ACT_GELU) return g * (0.5f * erfcf(-g * 0.70710678118654752f));
    const float s = 1.0f / (1.0f + expf(-g));
    return act == ACT_SIGMOID ? s : g * s;
}
__device__ __forceinline__ void act_both(int act, float g, float &a, float &da)
{
    if (act == ACT_RELU) {
        a = fmaxf(g, 0.0f);
        da = g > 0.0f ? 1.0f : 0.0f;
    } else if (act == ACT_GELU) {
        const float cdf = 0.5f * erfcf(-g * 0.70710678118654752f);
        a = g * cdf;
        da = cdf + g * expf(-0.5f * g * g) * 0.39894228040143268f;
    } else {
        const float s = 1.0f / (1.0f + expf(-g));
        a = act == ACT_SIGMOID ? s : g * s;
        da = act == ACT_SIGMOID ? s * (1.0f - s) : s * (1.0f + g * (1.0f - s));
    }
}

// Products on the float matrix cores (v_mfma_f32_32x32x2_f32, true float products), for any sizes: 128 x 128 of the output per block, a
// wave 64 x 64 of it, 16 of the contracted dimension at a time, two such tiles in LDS, the next one's loads in flight in registers.
constexpr int TILE = 128, DEPTH = 16;
// [row][k] tiles: 20 floats a row, so that the 16-byte reads of eight neighbouring rows lie on different banks
constexpr int PITCH = DEPTH + 4;

enum { NT_FORWARD, NT_GRAD };
struct NtArgs {
    const void *a, *b;        // [M][K], [N][K] (forward: [2N][K])
    int M, N, K;
    const float *bias;        // forward
    float *P;                 // forward: both projections [M][2N]
    void *out;                // h [M][N], or dx [M][N]
    const void *old, *gate;   // gradient epilogue
    int act;
};

template <class T, int MODE>
__global__ __launch_bounds__(TPB) void k_gated_nt(NtArgs p)
{
    __shared__ __align__(16) float lds[2][2][TILE][PITCH];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / 2, wn = wave % 2;
    const T *a = (const T *)p.a, *b = (const T *)p.b;
    constexpr int WIDE = MODE == NT_FORWARD ? TILE / 2 : TILE;
    const int across = (p.N + WIDE - 1) / WIDE, m0 = blockIdx.x / across * TILE, n0 = blockIdx.x % across * WIDE;
    // thread's elements: column tid % 16 of rows tid / 16 + 16 i
    const int k = tid % DEPTH, r0 = tid / DEPTH;
    constexpr int EACH = TILE * DEPTH / TPB;
    float ra[EACH], rb[EACH];
    auto weight_row = [&](int r) -> int {      // row of b behind row r of its tile, or -1
        if (MODE == NT_GRAD) return n0 + r < p.N ? n0 + r : -1;
        const int unit = n0 + r / 64 * 32 + r % 32;      // 32 units' gates, then the same units' linear parts
        return unit < p.N ? (r % 64 < 32 ? unit : p.N + unit) : -1;
    };
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int r = r0 + i * (TPB / DEPTH), wr = weight_row(r);
            const bool in = k0 + k < p.K;
            ra[i] = in && m0 + r < p.M ? to_f32(a[(size_t)(m0 + r) * p.K + k0 + k]) : 0.0f;
            rb[i] = in && wr >= 0 ? to_f32(b[(size_t)wr * p.K + k0 + k]) : 0.0f;
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            lds[buf][0][r0 + i * (TPB / DEPTH)][k] = ra[i];
            lds[buf][1][r0 + i * (TPB / DEPTH)][k] = rb[i];
        }
    };
    f32x16 acc[2][2] = {};
    const int steps = (p.K + DEPTH - 1) / DEPTH;
    load(0);
    store(0);
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
        if (s + 1 < steps) load((s + 1) * DEPTH);
        const int buf = s & 1;
#pragma unroll
        for (int q = 0; q < DEPTH / 8; ++q) {
            // the two halves of a wave take k and k + 4 of each product's pair
            const int kk = q * 8 + lane / 32 * 4;
            float4 fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fa[i] = *reinterpret_cast<const float4 *>(&lds[buf][0][wm * 64 + i * 32 + lane % 32][kk]);
                fb[i] = *reinterpret_cast<const float4 *>(&lds[buf][1][wn * 64 + i * 32 + lane % 32][kk]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i].x, fb[j].x, acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i].y, fb[j].y, acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i].z, fb[j].z, acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i].w, fb[j].w, acc[i][j], 0, 0, 0);
                }
        }
        if (s + 1 < steps) store(buf ^ 1);
    }
    // register r of lane l: row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = m0 + wm * 64 + i * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
            if (row >= p.M) continue;
            if (MODE == NT_FORWARD) {
                const int unit = n0 + wn * 32 + lane % 32;
                if (unit >= p.N) continue;
                const float g = acc[i][0][r] + (p.bias ? p.bias[unit] : 0.0f), u = acc[i][1][r] + (p.bias ? p.bias[p.N + unit] : 0.0f);
                float *P = p.P + (size_t)row * 2 * p.N + unit;
                P[0] = g;
                P[p.N] = u;
                ((T *)p.out)[(size_t)row * p.N + unit] = from_f32<T>(act_value(p.act, g) * u);
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = n0 + wn * 64 + j * 32 + lane % 32;
                    if (col >= p.N) continue;
                    const size_t at = (size_t)row * p.N + col;
                    const T *old = (const T *)p.old, *gate = (const T *)p.gate;
                    ((T *)p.out)[at] = grad_out<T>(acc[i][j][r], old != nullptr, old ? old[at] : from_f32<T>(0.0f), gate != nullptr,
                                                   gate ? gate[at] : from_f32<T>(0.0f));
                }
            }
        }
}

// dw[M][N] += a^T b with a [rows][M], b [rows][N], over the rows of split blockIdx.y; with several splits part[split][M][N] = their sums
template <class T>
__global__ __launch_bounds__(TPB) void k_gated_tn(const T *__restrict__ a, const T *__restrict__ b, int rows, int M, int N, int rows_per_split,
                                                  float *dw, float *part)
{
    __shared__ __align__(16) float lds[2][2][DEPTH][TILE];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / 2, wn = wave % 2;
    const int across = (N + TILE - 1) / TILE, m0 = blockIdx.x / across * TILE, n0 = blockIdx.x % across * TILE;
    const int first = blockIdx.y * rows_per_split, last = first + rows_per_split < rows ? first + rows_per_split : rows;
    const int c = tid % TILE, r0 = tid / TILE;
    constexpr int EACH = TILE * DEPTH / TPB;
    float ra[EACH], rb[EACH];
    auto load = [&](int at) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int r = at + r0 + i * (TPB / TILE);
            ra[i] = r < last && m0 + c < M ? to_f32(a[(size_t)r * M + m0 + c]) : 0.0f;
            rb[i] = r < last && n0 + c < N ? to_f32(b[(size_t)r * N + n0 + c]) : 0.0f;
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            lds[buf][0][r0 + i * (TPB / TILE)][c] = ra[i];
            lds[buf][1][r0 + i * (TPB / TILE)][c] = rb[i];
        }
    };
    f32x16 acc[2][2] = {};
    const int steps = (last - first + DEPTH - 1) / DEPTH;
    load(first);
    store(0);
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
        if (s + 1 < steps) load(first + (s + 1) * DEPTH);
        const int buf = s & 1;
#pragma unroll
        for (int q = 0; q < DEPTH / 2; ++q) {
            const int kk = q * 2 + lane / 32;
            float fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fa[i] = lds[buf][0][kk][wm * 64 + i * 32 + lane % 32];
                fb[i] = lds[buf][1][kk][wn * 64 + i * 32 + lane % 32];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
        if (s + 1 < steps) store(buf ^ 1);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = m0 + wm * 64 + i * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
            if (row >= M) continue;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int col = n0 + wn * 64 + j * 32 + lane % 32;
                if (col >= N) continue;
                if (part) part[((size_t)blockIdx.y * M + row) * N + col] = acc[i][j][r];
                else dw[(size_t)row * N + col] += acc[i][j][r];
            }
        }
}

// dw[i] += the sums of all splits, in their order
__global__ __launch_bounds__(TPB) void k_gated_tn_join(const float *__restrict__ part, int splits, size_t n, float *dw)
{
    const size_t i = (size_t)blockIdx.x * TPB + threadIdx.x;
    if (i >= n) return;
    float sum = 0.0f;
    for (int k = 0; k < splits; ++k) sum += part[(size_t)k * n + i];
    dw[i] += sum;
}

// Projections of four units from the sums of a product whose K was in `splits` parts, part[split][rows][2F]; F a multiple of 4
__global__ __launch_bounds__(TPB) void k_gated_join(const float *__restrict__ part, int splits, const float *__restrict__ bias, float *__restrict__ P,
                                                    bf16_t *__restrict__ h, int rows, int F, int act)
{
    const size_t i = ((size_t)blockIdx.x * TPB + threadIdx.x) * 4, n = (size_t)rows * F;
    if (i >= n) return;
    const size_t row = i / F, at = row * 2 * F + (i - row * F);
    const int unit = (int)(i - row * F);
    float4 g = make_float4(0.f, 0.f, 0.f, 0.f), u = g;
    auto add = [](float4 &t, const float *from) {
        const float4 v = *reinterpret_cast<const float4 *>(from);
        t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
    };
    for (int k = 0; k < splits; ++k) {
        add(g, part + (size_t)k * 2 * n + at);
        add(u, part + (size_t)k * 2 * n + at + F);
    }
    if (bias) {
        add(g, bias + unit);
        add(u, bias + F + unit);
    }
    *reinterpret_cast<float4 *>(P + at) = g;
    *reinterpret_cast<float4 *>(P + at + F) = u;
    uint2 v;
    v.x = pack_bf16(act_value(act, g.x) * u.x, act_value(act, g.y) * u.y);
    v.y = pack_bf16(act_value(act, g.z) * u.z, act_value(act, g.w) * u.w);
    *reinterpret_cast<uint2 *>(h + i) = v;
}

// D from dh and the projections, V units a thread (F a multiple of V, dh aligned to V elements)
template <class T, int V>
__global__ __launch_bounds__(TPB) void k_gated_grad(const T *__restrict__ dh, const float *__restrict__ P, T *__restrict__ D, size_t n, int F, int act)
{
    const size_t i = ((size_t)blockIdx.x * TPB + threadIdx.x) * V;
    if (i >= n) return;
    const size_t row = i / F, at = row * 2 * F + (i - row * F);
    typedef vec_t<T, V> vec;
    typedef vec_t<float, V> vecf;
    const vec d = *reinterpret_cast<const vec *>(dh + i);
    const vecf g = *reinterpret_cast<const vecf *>(P + at), u = *reinterpret_cast<const vecf *>(P + at + F);
    vec dg, du;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float a, da;
        act_both(act, g.e[j], a, da);
        const float v = to_f32(d.e[j]);
        dg.e[j] = from_f32<T>(v * u.e[j] * da);
        du.e[j] = from_f32<T>(v * a);
    }
    *reinterpret_cast<vec *>(D + at) = dg;
    *reinterpret_cast<vec *>(D + at + F) = du;
}

struct TnPlan {
    int splits, rows_per_split;
};
// two blocks for every unit, splits of 256 rows at the least
TnPlan tn_plan(int rows, int M, int N)
{
    const long long tiles = (long long)((M + TILE - 1) / TILE) * ((N + TILE - 1) / TILE);
    long long splits = 512 / tiles;
    const long long most = (rows + 255) / 256;
    splits = splits < 1 ? 1 : splits > most ? most : splits;
    TnPlan p;
    p.rows_per_split = (int)((rows + splits - 1) / splits);
    p.splits = (rows + p.rows_per_split - 1) / p.rows_per_split;
    return p;
}

}  // namespace

// every row a map of one pixel
static GatherConv rows_product(int rows, int ci, int co, bool panels)
{
    GatherConv g;
    g.N = rows;
    g.Hi = g.Wi = g.Ho = g.Wo = g.R = g.S = g.s_out = g.s_in = 1;
    g.pad_h = g.pad_w = 0;
    g.Ci = ci;
    g.Co = co;
    g.wt_panels = panels;
    return g;
}

bool gated_mfma(int dt, int rows, int C, int F)
{
    return dt == DT_BF16 && F % 8 == 0 && conv_gather_mfma_supported(rows_product(rows, C, 2 * F, false)) &&
           conv_gather_mfma_supported(rows_product(rows, 2 * F, C, false)) && conv_wgrad_mfma_supported({rows, 1, 1, C, 1, 1, 2 * F, 1, 1, 1, 0});
}

size_t gated_workspace(int dt, int rows, int C, int F)
{
    if (gated_mfma(dt, rows, C, F)) return conv_gather_mfma_raw_workspace(rows_product(rows, C, 2 * F, false));
    const TnPlan p = tn_plan(rows, 2 * F, C);
    const size_t part = p.splits > 1 ? (size_t)p.splits * 2 * F * C * sizeof(float) : 0, sums = colsum_workspace(rows, 2 * F);
    return part > sums ? part : sums;
}

#define GATED_T(dt, ...)                                              \
    do {                                                              \
        if ((dt) == DT_F32) { using T = float; __VA_ARGS__; }         \
        else { using T = bf16_t; __VA_ARGS__; }                       \
    } while (0)

hipError_t gated_fwd(int dt, int act, const void *x, const void *w, const float *bias, float *P, void *h, int rows, int C, int F, bool panels,
                     void *workspace, hipStream_t s)
{
    if (gated_mfma(dt, rows, C, F)) {
        int splits = 0;
        const hipError_t e = conv_gather_mfma_raw(x, w, rows_product(rows, C, 2 * F, panels), (float *)workspace, &splits, s);
        if (e != hipSuccess) return e;
        const size_t n = (size_t)rows * F / 4;
        hipLaunchKernelGGL(k_gated_join, dim3((unsigned)((n + TPB - 1) / TPB)), dim3(TPB), 0, s, (const float *)workspace, splits, bias, P, (bf16_t *)h,
                           rows, F, act);
        return hipGetLastError();
    }
    if (panels) return hipErrorInvalidValue;
    NtArgs a{x, w, rows, F, C, bias, P, h, nullptr, nullptr, act};
    const dim3 grid((unsigned)((F + TILE / 2 - 1) / (TILE / 2)) * ((rows + TILE - 1) / TILE));
    GATED_T(dt, hipLaunchKernelGGL((k_gated_nt<T, NT_FORWARD>), grid, dim3(TPB), 0, s, a));
    return hipGetLastError();
}

hipError_t gated_grad(int dt, int act, const void *dh, const float *P, void *D, int rows, int F, hipStream_t s)
{
    const size_t n = (size_t)rows * F;
    const bool four = F % 4 == 0 && (uintptr_t)dh % (4 * dt_size(dt)) == 0;      // the caller's dh may lie anywhere
    const dim3 grid((unsigned)((n / (four ? 4 : 1) + TPB - 1) / TPB));
    if (four) GATED_T(dt, hipLaunchKernelGGL((k_gated_grad<T, 4>), grid, dim3(TPB), 0, s, (const T *)dh, P, (T *)D, n, F, act));
    else GATED_T(dt, hipLaunchKernelGGL((k_gated_grad<T, 1>), grid, dim3(TPB), 0, s, (const T *)dh, P, (T *)D, n, F, act));
    return hipGetLastError();
}

hipError_t gated_dgrad_direct(int dt, const void *D, const void *wt, void *dx, GradEpi epi, int rows, int C, int F, hipStream_t s)
{
    const void *old = epi.accum ? (epi.accum_from ? epi.accum_from : dx) : nullptr;
    NtArgs a{D, wt, rows, C, 2 * F, nullptr, nullptr, dx, old, epi.gate, 0};
    const dim3 grid((unsigned)((C + TILE - 1) / TILE) * ((rows + TILE - 1) / TILE));
    GATED_T(dt, hipLaunchKernelGGL((k_gated_nt<T, NT_GRAD>), grid, dim3(TPB), 0, s, a));
    return hipGetLastError();
}

hipError_t gated_wgrad_direct(int dt, const void *x, const void *D, float *dw, float *db, int rows, int C, int F, void *workspace, hipStream_t s)
{
    const int M = 2 * F;
    const TnPlan p = tn_plan(rows, M, C);
    float *part = p.splits > 1 ? (float *)workspace : nullptr;
    const dim3 grid((unsigned)((C + TILE - 1) / TILE) * ((M + TILE - 1) / TILE), p.splits);
    GATED_T(dt, hipLaunchKernelGGL((k_gated_tn<T>), grid, dim3(TPB), 0, s, (const T *)D, (const T *)x, rows, M, C, p.rows_per_split, dw, part));
    if (part) {
        const size_t n = (size_t)M * C;
        hipLaunchKernelGGL(k_gated_tn_join, dim3((unsigned)((n + TPB - 1) / TPB)), dim3(TPB), 0, s, part, p.splits, n, dw);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !db) return e;
    return colsum_accumulate(dt, D, rows, M, db, workspace, s);
}

}  // namespace bapipe
