// Layer norm over the channels of every position of an NHWC tensor, read as a matrix [rows][C].
//   mean = sum x / C, var = sum (x - mean)^2 / C, inv = 1 / sqrt(var + eps), xhat = (x - mean) inv, y = gamma xhat + beta
//   a = gamma dy;  dx = inv (a - sum a / C - xhat sum(a xhat) / C);  dgamma += sum over rows of dy xhat;  dbeta += sum over rows of dy
// Everything between a load and a store is float; mean and inv of every row are kept for the backward pass.
//
// HBM bounds it: forward reads x and writes y, backward reads x and dy and writes dx, each once.  A row stays in the registers of
// the threads that read it, so that its variance is taken around its own mean (E[x^2] - mean^2 of rows far from zero loses
// all digits) without a second read.  A group of threads takes one row after another and keeps what belongs to its columns,
// gamma and beta, or gamma and the sums of the columns' gradients: read for every row, the two floats of a bf16 element are twice
// the bytes of the element's load and store.  The next row is requested before the present one's sums are formed.
#include "kernels.h"
#include "mfma_common.h"

namespace bapipe {
namespace {

constexpr int TPB = 256;

// ------------------------------------------------------------------ sums over the threads of a row
// Of a wave: neighbours by data-parallel moves inside the vector unit, without LDS, the total broadcast from the last lane
__device__ __forceinline__ float wave_total(float v)
{
    auto add = [&](auto moved) { v += __int_as_float(moved); };
#define MOVED(ctrl, rows) __builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xF, true)
    add(MOVED(0x111, 0xF));        // from the lane 1, 2, 4, 8 below, inside rows of 16 lanes
    add(MOVED(0x112, 0xF));
    add(MOVED(0x114, 0xF));
    add(MOVED(0x118, 0xF));
    add(MOVED(0x142, 0xA));        // the last lane of a row to the row behind it, 0 to 1 and 2 to 3
    add(MOVED(0x143, 0xC));        // and of the lower half to the upper one
#undef MOVED
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Of the G threads of a group, for all of them.  Groups of 256 exchange their waves' totals in lds[2][WAVES]; two calls in turn use
// different halves, so that one barrier a call is enough.
template <int G>
__device__ __forceinline__ float group_sum(float v, float *lds, int half)
{
    if constexpr (G < 64) {
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, G);
        return v;
    } else {
        v = wave_total(v);
        if constexpr (G == 64) return v;
        constexpr int W = G / 64;
        float *mine = lds + (half * (blockDim.x / 64)) + threadIdx.x / G * W;
        if (threadIdx.x % 64 == 0) mine[threadIdx.x / 64 % W] = v;
        __syncthreads();
        float sum = mine[0];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += mine[w];
        return sum;
    }
}

// The thread's group in its block, known to be the same for a wave where it is: a row's address is then none of its registers'
template <int G> __device__ __forceinline__ int group_of()
{
    const int group = threadIdx.x / G;
    return G >= 64 ? __builtin_amdgcn_readfirstlane(group) : group;
}

// ------------------------------------------------------------------ rows that fit their threads' registers
// V = 16 / sizeof(T) values in one access at any address of T (global memory needs no more alignment than that); where a row
// is no whole number of them (TAIL), the last ones of it are `left` < V single values, and zeros behind them
template <class T, int V> struct vec_of {
    T e[V];
};
template <bool TAIL, class T, int V> __device__ __forceinline__ void load_vec(vec_of<T, V> &to, const T *from, int left)
{
    if (!TAIL || left >= V) {
        __builtin_memcpy(&to, from, sizeof(to));
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) to.e[j] = j < left ? from[j] : T{};
}
template <bool TAIL, class T, int V> __device__ __forceinline__ void store_vec(T *to, const vec_of<T, V> &from, int left)
{
    if (!TAIL || left >= V) {
        __builtin_memcpy(to, &from, sizeof(from));
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j < left) to[j] = from.e[j];
}

// Values of T stay packed as they were read: taken apart, two bf16 would be two registers
template <bool TAIL, class T> __device__ __forceinline__ chunk16 load_packed(const T *from, int left)
{
    vec_of<T, 16 / sizeof(T)> v;
    load_vec<TAIL>(v, from, left);
    return __builtin_bit_cast(chunk16, v);
}

// Thread t of a group of G has columns (k G + t) V .. + V - 1, k < NV.
template <class T, int NV> struct row_regs {
    static constexpr int V = 16 / sizeof(T);
    chunk16 v[NV];
    template <int G, bool TAIL> __device__ __forceinline__ void load(const T *row, int t, int C)
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + t) * V;
            v[k] = chunk16{0u, 0u, 0u, 0u};
            if (c < C) v[k] = load_packed<TAIL>(row + c, C - c);
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] = chunk16{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ float at(int k, int j) const { return chunk_value<T>(v[k], j); }
    // what was computed from the values so far is not to be kept for later
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) asm volatile("" : "+v"(v[k]));
    }
};
template <int V, int NV> struct column_regs {
    vec_of<float, V> v[NV];
    template <int G, bool TAIL> __device__ __forceinline__ void load(const float *row, int t, int C)
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) v[k].e[j] = 0.0f;
            if (c < C) load_vec<TAIL>(v[k], row + c, C - c);
        }
    }
};

template <class T> struct FwdArgs {
    const T *x;
    const float *gamma, *beta;
    T *y, *copy, *rest;       // copy: x once more, rest: what rounding took from y, each NULL or [rows][C]
    float *stats, eps;
    int rows, C;
};

template <class T, int NV, int G, bool TAIL>
__global__ __launch_bounds__(G > TPB ? G : TPB) void k_layernorm_fwd(FwdArgs<T> p)
{
    constexpr int V = 16 / sizeof(T), GROUPS = G > TPB ? 1 : TPB / G;
    __shared__ float lds[2 * GROUPS * G / 64];
    const int t = threadIdx.x % G, C = p.C, step = gridDim.x * GROUPS;
    int row = blockIdx.x * GROUPS + group_of<G>();
    column_regs<V, NV> gamma, beta;
    gamma.template load<G, TAIL>(p.gamma, t, C);
    beta.template load<G, TAIL>(p.beta, t, C);
    row_regs<T, NV> next;
    if (row < p.rows) next.template load<G, TAIL>(p.x + (size_t)row * C, t, C);
    const float per = 1.0f / C;
    // columns behind the row's end
    auto in = [&](int k, int j) { return (k * G + t) * V + (TAIL ? j : 0) < C; };
    // all groups of a block take the same number of turns, for they meet at barriers
    for (int first = blockIdx.x * GROUPS; first < p.rows; first += step, row += step) {
        const bool on = row < p.rows;
        const row_regs<T, NV> x = next;
        if (row + step < p.rows) next.template load<G, TAIL>(p.x + (size_t)(row + step) * C, t, C);
        float f[NV][V], sum = 0.0f, sq = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                f[k][j] = in(k, j) ? x.at(k, j) : 0.0f;
                sum += f[k][j];
            }
        const float mean = group_sum<G>(sum, lds, 0) * per;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                f[k][j] = in(k, j) ? f[k][j] - mean : 0.0f;
                sq = fmaf(f[k][j], f[k][j], sq);
            }
        const float inv = 1.0f / sqrtf(group_sum<G>(sq, lds, 1) * per + p.eps);
        if (!on) continue;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + t) * V;
            if (c >= C) continue;
            const size_t at = (size_t)row * C + c;
            vec_of<T, V> y, rest;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float v = fmaf(f[k][j] * inv, gamma.v[k].e[j], beta.v[k].e[j]);
                y.e[j] = from_f32<T>(v);
                if (p.rest) rest.e[j] = from_f32<T>(rounding_took(v, to_f32(y.e[j])));
            }
            store_vec<TAIL>(p.y + at, y, C - c);
            if (p.rest) store_vec<TAIL>(p.rest + at, rest, C - c);
            if (p.copy) store_vec<TAIL>(p.copy + at, __builtin_bit_cast(vec_of<T, V>, x.v[k]), C - c);
        }
        if (t == 0) {
            p.stats[row] = mean;
            p.stats[p.rows + row] = inv;
        }
    }
}

template <class T> struct BwdArgs {
    const T *x, *dy;
    const float *dy_parts;    // instead of dy: its `parts` float sums [parts][rows][C]
    int parts;
    const float *gamma, *stats;
    T *dx;                    // may be NULL, or dy
    const T *old, *gate;
    float *part;              // [gridDim.x][2][C]: sums over the block's rows of dy xhat and of dy
    float *dgamma, *dbeta;    // where a lone block adds its own
    int rows, C;
};

// Floats from one group's columns' sums in LDS to the next one's: groups that share a wave write to different banks
constexpr int meet_pitch(int nv, int v, int g) { return nv * v * 2 * g + (g < 64 ? g : 0); }
// Whether gamma stays in LDS, behind the words that the waves' totals take: where sums, values and gamma of 16 columns are a few registers more
// than the 128 with which two blocks fit a unit.  Spilled, those were 24 KB of a row of 8192 beside its own 49 KB (bf16, 16384 rows: 208
// us, so 175; 8192 rows of 5000: 109 and 73).  Floats, 8 columns, fit (8192 rows of 4096: 84, so 86); with what an epilogue adds it is
// one block either way.
constexpr bool shared_gamma(int nv, int v, int g, bool epi) { return nv * v == 16 && g >= 256 && !epi; }
constexpr int kGammaAt = 64;

// NT threads, NT / G groups whose columns' sums meet in LDS at the end.  (In three rounds of halves, with the sums of a thread's columns
// side by side, 3200 rows of 1024 bf16 took 15.8 us instead of 11.7.)
// A row is taken from its packed values twice, for the sums and for dx: kept as floats in between, two rows of them, it cost twice
// the registers, and rows of 8192 spilled (16384 of them, bf16: 341 us where the 805 MB of x, dy and dx take 155 at the copy's rate).
template <class T, int NV, int G, int NT, bool TAIL, bool PARTS, bool EPI>
__global__ __launch_bounds__(NT, NV == 1 || (NV == 2 && !EPI) ? 4 : 2) void k_layernorm_bwd(BwdArgs<T> p)
{
    extern __shared__ __align__(16) float lds[];
    constexpr int V = 16 / sizeof(T), GROUPS = NT / G;
    const int t = threadIdx.x % G, group = group_of<G>(), C = p.C, step = gridDim.x * GROUPS;
    int row = blockIdx.x * GROUPS + group;
    constexpr bool SHARED = shared_gamma(NV, V, G, EPI);
    float *const gamma_lds = lds + kGammaAt;
    column_regs<V, NV> gamma;
    gamma.template load<G, TAIL>(p.gamma, t, C);
    if constexpr (SHARED) {
        if (group == 0)
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int q = 0; q < V / 4; ++q) __builtin_memcpy(gamma_lds + ((k * (V / 4) + q) * G + t) * 4, &gamma.v[k].e[q * 4], 16);
        __syncthreads();
    }
    auto gammas = [&](int k) {
        if constexpr (!SHARED) return gamma.v[k];
        vec_of<float, V> g;
#pragma unroll
        for (int q = 0; q < V / 4; ++q) __builtin_memcpy(&g.e[q * 4], gamma_lds + ((k * (V / 4) + q) * G + t) * 4, 16);
        return g;
    };
    float sg[NV][V] = {}, sb[NV][V] = {};
    row_regs<T, NV> nx, nd;
    float nmean = 0.0f, ninv = 0.0f;
    auto request = [&](int r) {
        nmean = p.stats[r];
        ninv = p.stats[p.rows + r];
        nx.template load<G, TAIL>(p.x + (size_t)r * C, t, C);
        if (!PARTS) nd.template load<G, TAIL>(p.dy + (size_t)r * C, t, C);
    };
    nx.clear();
    nd.clear();
    if (row < p.rows) request(row);
    const float per = 1.0f / C;
    for (int first = blockIdx.x * GROUPS; first < p.rows; first += step, row += step) {
        const bool on = row < p.rows;
        row_regs<T, NV> x = nx, dy = nd;
        const float mean = nmean, inv = ninv;
        if (row + step < p.rows) request(row + step);
        else {                                           // behind its last row a group adds nothing to anything
            nmean = ninv = 0.0f;
            nx.clear();
            nd.clear();
        }
        const size_t base = (size_t)row * C;
        float sums[PARTS ? NV : 1][V];
        if constexpr (PARTS) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = (k * G + t) * V;
#pragma unroll
                for (int j = 0; j < V; ++j) sums[k][j] = 0.0f;
                if (on && c < C)
                    for (int s = 0; s < p.parts; ++s) {
                        vec_of<float, V> v;
                        load_vec<TAIL>(v, p.dy_parts + (size_t)s * p.rows * C + base + c, C - c);
#pragma unroll
                        for (int j = 0; j < V; ++j) sums[k][j] += v.e[j];
                    }
            }
        }
        // dy and xhat of a column; behind the row's end dy is 0
        auto column = [&](int k, int j, float &d, float &xh) {
            d = PARTS ? sums[PARTS ? k : 0][j] : dy.at(k, j);
            xh = (x.at(k, j) - mean) * inv;
        };
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const vec_of<float, V> ga = gammas(k);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float d, xh;
                column(k, j, d, xh);
                const float dx = d * xh, g = ga.e[j];
                sg[k][j] += dx;
                sb[k][j] += d;
                s1 = fmaf(d, g, s1);
                s2 = fmaf(dx, g, s2);
            }
            __builtin_amdgcn_sched_barrier(0);           // one access's columns at a time, or all of them are in registers at once
        }
        if (!p.dx) continue;
        s1 = group_sum<G>(s1, lds, 0) * per;
        s2 = group_sum<G>(s2, lds, 1) * per;
        if (!on) continue;
        x.forget();
        dy.forget();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + t) * V;
            if (c >= C) continue;
            const vec_of<float, V> ga = gammas(k);
            vec_of<T, V> r;
            chunk16 old, gate;
            if (EPI && p.old) old = load_packed<TAIL>(p.old + base + c, C - c);
            if (EPI && p.gate) gate = load_packed<TAIL>(p.gate + base + c, C - c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float d, xh;
                column(k, j, d, xh);
                const float v = inv * (d * ga.e[j] - s1 - xh * s2);
                if constexpr (!EPI) r.e[j] = from_f32<T>(v);
                else
                    r.e[j] = grad_out<T>(v, p.old != nullptr, from_f32<T>(p.old ? chunk_value<T>(old, j) : 0.0f), p.gate != nullptr,
                                         from_f32<T>(p.gate ? chunk_value<T>(gate, j) : 0.0f));
            }
            store_vec<TAIL>(p.dx + base + c, r, C - c);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    float *to = p.part + (size_t)blockIdx.x * 2 * C;
    const bool lone = gridDim.x == 1;
    if constexpr (GROUPS == 1) {
        // whole accesses: one float after another, 32 bytes apart across the threads, took 175 us instead of 162 at 16384 rows of 8192
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + t) * V;
            if (c >= C) continue;
            vec_of<float, V> g, b;
            if (lone) {
                load_vec<TAIL>(g, p.dgamma + c, C - c);
                load_vec<TAIL>(b, p.dbeta + c, C - c);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                g.e[j] = (lone ? g.e[j] : 0.0f) + sg[k][j];
                b.e[j] = (lone ? b.e[j] : 0.0f) + sb[k][j];
            }
            store_vec<TAIL>(lone ? p.dgamma + c : to + c, g, C - c);
            store_vec<TAIL>(lone ? p.dbeta + c : to + C + c, b, C - c);
        }
    } else {
        // a group's sums in the order access, value, gamma or beta, thread, a value's threads turned by 64 / V places from one value to the next:
        // neighbours write the sums of one value and read those of neighbouring columns, either from different banks
        constexpr int N = NV * V * 2 * G, PITCH = meet_pitch(NV, V, G);
        auto place = [](int k, int j, int beta, int t) { return ((k * V + j) * 2 + beta) * G + (t ^ (j * (64 / V) & (G - 1))); };
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                lds[group * PITCH + place(k, j, 0, t)] = sg[k][j];
                lds[group * PITCH + place(k, j, 1, t)] = sb[k][j];
            }
        __syncthreads();
        for (int v = threadIdx.x; v < N; v += NT) {
            const int j = v % V, u = v / V % G, beta = v / V / G % 2, k = v / V / G / 2, c = (k * G + u) * V + j;
            float sum = 0.0f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) sum += lds[g * PITCH + place(k, j, beta, u)];
            if (c >= C) continue;
            if (lone) (beta ? p.dbeta : p.dgamma)[c] += sum;
            else to[beta * C + c] = sum;
        }
    }
}

// ------------------------------------------------------------------ longer rows, read once for every sum
__device__ __forceinline__ float block_sum(float v, float *lds)
{
    v = wave_total(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < TPB / 64; ++w) sum += lds[w];
    return sum;
}

template <class T>
__global__ __launch_bounds__(TPB) void k_layernorm_fwd_long(FwdArgs<T> p)
{
    __shared__ float lds[TPB / 64];
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const size_t at = (size_t)row * p.C;
        float sum = 0.0f, sq = 0.0f;
        for (int c = threadIdx.x; c < p.C; c += TPB) sum += to_f32(p.x[at + c]);
        const float mean = block_sum(sum, lds) / p.C;
        for (int c = threadIdx.x; c < p.C; c += TPB) {
            const float d = to_f32(p.x[at + c]) - mean;
            sq += d * d;
        }
        const float inv = 1.0f / sqrtf(block_sum(sq, lds) / p.C + p.eps);
        for (int c = threadIdx.x; c < p.C; c += TPB) {
            const float v = fmaf((to_f32(p.x[at + c]) - mean) * inv, p.gamma[c], p.beta[c]);
            const T y = from_f32<T>(v);
            if (p.rest) p.rest[at + c] = from_f32<T>(rounding_took(v, to_f32(y)));
            if (p.copy) p.copy[at + c] = p.x[at + c];
            p.y[at + c] = y;
        }
        if (threadIdx.x == 0) {
            p.stats[row] = mean;
            p.stats[p.rows + row] = inv;
        }
    }
}

template <class T> __device__ __forceinline__ float dy_at(const BwdArgs<T> &p, size_t i)
{
    if (!p.dy_parts) return to_f32(p.dy[i]);
    float v = 0.0f;
    for (int s = 0; s < p.parts; ++s) v += p.dy_parts[(size_t)s * p.rows * p.C + i];
    return v;
}

template <class T>
__global__ __launch_bounds__(TPB) void k_layernorm_dx_long(BwdArgs<T> p)
{
    __shared__ float lds[TPB / 64];
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const size_t at = (size_t)row * p.C;
        const float mean = p.stats[row], inv = p.stats[p.rows + row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x; c < p.C; c += TPB) {
            const float a = dy_at(p, at + c) * p.gamma[c];
            s1 += a;
            s2 += a * ((to_f32(p.x[at + c]) - mean) * inv);
        }
        s1 = block_sum(s1, lds) / p.C;
        s2 = block_sum(s2, lds) / p.C;
        for (int c = threadIdx.x; c < p.C; c += TPB) {
            const float a = dy_at(p, at + c) * p.gamma[c], xhat = (to_f32(p.x[at + c]) - mean) * inv;
            p.dx[at + c] = grad_out<T>(inv * (a - s1 - xhat * s2), p.old != nullptr, p.old ? p.old[at + c] : from_f32<T>(0.0f), p.gate != nullptr,
                                       p.gate ? p.gate[at + c] : from_f32<T>(0.0f));
        }
    }
}

// part[chunk][0 | 1][C]: sums of dy xhat and of dy over the chunk's rows, a column per thread
template <class T>
__global__ __launch_bounds__(TPB) void k_layernorm_columns(BwdArgs<T> p, int rows_per_chunk)
{
    const int c = blockIdx.x * TPB + threadIdx.x;
    if (c >= p.C) return;
    const int r0 = blockIdx.y * rows_per_chunk, r1 = r0 + rows_per_chunk < p.rows ? r0 + rows_per_chunk : p.rows;
    float g = 0.0f, b = 0.0f;
    for (int r = r0; r < r1; ++r) {
        const float d = dy_at(p, (size_t)r * p.C + c);
        g += d * ((to_f32(p.x[(size_t)r * p.C + c]) - p.stats[r]) * p.stats[p.rows + r]);
        b += d;
    }
    p.part[(size_t)blockIdx.y * 2 * p.C + c] = g;
    p.part[((size_t)blockIdx.y * 2 + 1) * p.C + c] = b;
}

// dgamma += , dbeta += the sums of all chunks: 16 columns a block, 16 threads each that take every 16th chunk and are added in
// their order
__global__ __launch_bounds__(TPB) void k_layernorm_params(const float *__restrict__ part, int chunks, int C, float *dgamma, float *dbeta)
{
    __shared__ float lds[16][17];
    const int col = threadIdx.x % 16, lane = threadIdx.x / 16;
    const long long i = (long long)blockIdx.x * 16 + col, n = 2ll * C;
    float sum = 0.0f;
    if (i < n) {
        int k = lane;
        for (; k + 48 < chunks; k += 64) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = part[(size_t)(k + 16 * u) * n + i];
            sum += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; k < chunks; k += 16) sum += part[(size_t)k * n + i];
    }
    lds[lane][col] = sum;
    __syncthreads();
    if (lane || i >= n) return;
    float total = 0.0f;
#pragma unroll
    for (int u = 0; u < 16; ++u) total += lds[u][col];
    float *out = i < C ? dgamma + i : dbeta + (i - C);
    *out += total;
}

// ------------------------------------------------------------------ which kernel takes a row
// G threads and NV accesses of each for a row, the smallest that fit it: a wave for a row of up to 4 a thread (forward) or 2 (backward,
// which has two rows of registers and two sums for every column: of 4 it spills), then four and eight waves.  G = 0: too long for registers.
struct Shape {
    int nv, g;
};
Shape shape_of(int dt, int C, bool fwd)
{
    const int v = dt == DT_F32 ? 4 : 8, n = (C + v - 1) / v;
    static const Shape forward[] = {{1, 8}, {1, 16}, {1, 32}, {1, 64}, {2, 64}, {4, 64}, {2, 256}, {4, 256}, {4, 512}};
    static const Shape backward[] = {{1, 8}, {1, 16}, {1, 32}, {1, 64}, {2, 64}, {1, 256}, {2, 256}, {2, 512}, {4, 512}};
    for (const Shape &k : fwd ? forward : backward)
        if (n <= k.nv * k.g) return k;
    return {0, 0};
}

// Blocks of the backward pass: each leaves 8 C bytes of column sums for the kernel behind it, against 6 C bytes a row and more of its
// own, so that a block takes 32 rows where that leaves two for every unit; up to four rounds of one block's groups do without that kernel
int bwd_blocks(int rows, int groups)
{
    if (rows <= 4 * groups) return 1;
    const int all = (rows + groups - 1) / groups, long_ones = rows / 32, many = long_ones > 512 ? 512 : long_ones < 256 ? 256 : long_ones;
    return all < many ? all : many;
}
// Rows whose columns' sums a thread of the long rows' kernel adds up: at most 256 such chunks
int long_chunk(int rows)
{
    constexpr int most = 256;
    return rows < 64 * most ? 64 : (rows + most - 1) / most;
}
constexpr int kBwdThreads = 512;

}  // namespace

size_t layernorm_workspace(int dt, int rows, int C)
{
    const Shape k = shape_of(dt, C, false);
    const int blocks = k.g ? bwd_blocks(rows, kBwdThreads / k.g) : (rows + long_chunk(rows) - 1) / long_chunk(rows);
    return k.g && blocks == 1 ? 0 : (size_t)blocks * 2 * C * sizeof(float);      // a lone block adds its own
}

template <class T>
static hipError_t fwd_t(int dt, FwdArgs<T> p, hipStream_t s)
{
    const Shape k = shape_of(dt, p.C, true);
    const bool tail = p.C % (16 / sizeof(T)) != 0;
    auto launch = [&](auto kernel, int g) {
        const int groups = g > TPB ? 1 : TPB / g, blocks = (p.rows + groups - 1) / groups, most = 256 * 8;
        hipLaunchKernelGGL(kernel, dim3(blocks < most ? blocks : most), dim3(groups * g), 0, s, p);
        return hipGetLastError();
    };
#define FWD(NV, G)                                                                                  \
    if (k.nv == NV && k.g == G)                                                                     \
    return tail ? launch(k_layernorm_fwd<T, NV, G, true>, G) : launch(k_layernorm_fwd<T, NV, G, false>, G)
    FWD(1, 8); FWD(1, 16); FWD(1, 32); FWD(1, 64); FWD(2, 64); FWD(4, 64); FWD(2, 256); FWD(4, 256); FWD(4, 512);
#undef FWD
    const dim3 grid(p.rows < (1 << 20) ? p.rows : 1 << 20);
    hipLaunchKernelGGL(k_layernorm_fwd_long<T>, grid, dim3(TPB), 0, s, p);
    return hipGetLastError();
}

template <class T>
static hipError_t bwd_t(int dt, BwdArgs<T> p, hipStream_t s)
{
    const Shape k = shape_of(dt, p.C, false);
    const bool tail = p.C % (16 / sizeof(T)) != 0;
    int chunks = 0;
    const bool epi = p.old || p.gate;
    auto launch = [&](auto kernel, int threads, int groups) {
        chunks = bwd_blocks(p.rows, groups);
        const int v = 16 / (int)sizeof(T);
        const size_t meet = groups > 1 ? (size_t)groups * meet_pitch(k.nv, v, k.g) : 0;
        const size_t loop = shared_gamma(k.nv, v, k.g, epi) ? kGammaAt + (size_t)k.nv * v * k.g : 2 * threads / 64;
        const size_t bytes = (meet > loop ? meet : loop) * sizeof(float);        // at most 64 KB
        hipLaunchKernelGGL(kernel, dim3(chunks), dim3(threads), bytes, s, p);
        return hipGetLastError();
    };
    hipError_t e = hipErrorInvalidValue;
    bool found = false;
#define BWD_(NV, G, NT, TAIL, PARTS) \
    (epi ? launch(k_layernorm_bwd<T, NV, G, NT, TAIL, PARTS, true>, NT, NT / G) : launch(k_layernorm_bwd<T, NV, G, NT, TAIL, PARTS, false>, NT, NT / G))
#define BWD(NV, G)                                                                                                             \
    if (!found && k.nv == NV && k.g == G) {                                                                                    \
        found = true;                                                                                                          \
        if constexpr (sizeof(T) == 2) {                                                                                        \
            if (p.dy_parts) e = tail ? BWD_(NV, G, kBwdThreads, true, true) : BWD_(NV, G, kBwdThreads, false, true);           \
        }                                                                                                                      \
        if (!p.dy_parts) e = tail ? BWD_(NV, G, kBwdThreads, true, false) : BWD_(NV, G, kBwdThreads, false, false);            \
    }
    BWD(1, 8); BWD(1, 16); BWD(1, 32); BWD(1, 64); BWD(2, 64);
    BWD(1, 256); BWD(2, 256); BWD(2, 512); BWD(4, 512);
#undef BWD
#undef BWD_
    if (!found) {
        // the columns first, for dx may take the place of dy
        const int per = long_chunk(p.rows);
        chunks = (p.rows + per - 1) / per;
        hipLaunchKernelGGL(k_layernorm_columns<T>, dim3((p.C + TPB - 1) / TPB, chunks), dim3(TPB), 0, s, p, per);
        if (p.dx) hipLaunchKernelGGL(k_layernorm_dx_long<T>, dim3(p.rows < (1 << 20) ? p.rows : 1 << 20), dim3(TPB), 0, s, p);
        e = hipGetLastError();
    }
    if (e != hipSuccess || (found && chunks == 1)) return e;
    hipLaunchKernelGGL(k_layernorm_params, dim3((unsigned)((2ll * p.C + 15) / 16)), dim3(TPB), 0, s, p.part, chunks, p.C, p.dgamma, p.dbeta);
    return hipGetLastError();
}

hipError_t layernorm_fwd(int dt, const void *x, const float *gamma, const float *beta, float eps, void *y, float *stats, int rows, int C, hipStream_t s,
                         void *copy, void *rest)
{
    if (dt == DT_F32) return fwd_t<float>(dt, {(const float *)x, gamma, beta, (float *)y, (float *)copy, (float *)rest, stats, eps, rows, C}, s);
    return fwd_t<bf16_t>(dt, {(const bf16_t *)x, gamma, beta, (bf16_t *)y, (bf16_t *)copy, (bf16_t *)rest, stats, eps, rows, C}, s);
}

hipError_t layernorm_bwd(int dt, const void *x, const void *dy, int dy_parts, const float *gamma, const float *stats, void *dx, float *dgamma,
                         float *dbeta, GradEpi epi, int rows, int C, void *workspace, hipStream_t s)
{
    const void *old = epi.accum ? (epi.accum_from ? epi.accum_from : dx) : nullptr;
    const float *parts = dy_parts ? (const float *)dy : nullptr;
    if (parts) dy = nullptr;
    if (dt == DT_F32)
        return bwd_t<float>(dt, {(const float *)x, (const float *)dy, parts, dy_parts, gamma, stats, (float *)dx, (const float *)old, (const float *)epi.gate,
                                 (float *)workspace, dgamma, dbeta, rows, C}, s);
    return bwd_t<bf16_t>(dt, {(const bf16_t *)x, (const bf16_t *)dy, parts, dy_parts, gamma, stats, (bf16_t *)dx, (const bf16_t *)old,
                              (const bf16_t *)epi.gate, (float *)workspace, dgamma, dbeta, rows, C}, s);
}

}  // namespace bapipe
