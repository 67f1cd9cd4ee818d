// Gated linear layer, at every position (row) of an NHWC tensor:
//   [g | u] = x W^T + b, W [2F][C] with the F gate rows first;  h = act(g) u
//   D = [dh u act'(g) | dh act(g)];  dx = D W;  dW += D^T x;  db += sum over rows of D
// g and u are kept in float for the backward pass, P [rows][2F].  Rounded to bf16 they were, with D's own rounding, what a
// bf16 layer's gradients were off by most: 3.0e-3 of dW and dx against 64 bits (2-norm), 2.3e-3 so.
// Products of bf16 whose widths are multiples of 8 run on the bf16 matrix cores, the others on the float ones.
#include "kernels.h"
#include "mfma_common.h"
#include <type_traits>

namespace bapipe {
namespace {

constexpr int TPB = 256;
typedef f32x16_t f32x16;

// act(g), and its derivative.  A ReLU's derivative at 0 is 0, as everywhere in the library; of NaN its value is NaN.  A float layer takes the library's
// exp and erfc; for a bf16 one, whose results are rounded to 8 bits, the hardware's exp2 and reciprocal (a few 2^-24 off, times |g|)
// and, with t = 1 / (1 + 0.4 x), erfc(x) = exp(-x^2) t q(t), q a polynomial of degree 8 fitted here to erfcx(x) / t over
// x >= 0 for the least largest relative error: 2.8e-7 in float arithmetic, in the tail as well, where 1 + erf is all
// cancellation.  The library's erfc was a quarter of the forward kernel's time.
template <class T> constexpr bool kFast = sizeof(T) == 2;
template <bool FAST> __device__ __forceinline__ float exp_of(float x) { return FAST ? __builtin_amdgcn_exp2f(x * 1.44269504088896341f) : expf(x); }
template <bool FAST> __device__ __forceinline__ float sigmoid_of(float g)
{
    const float e = 1.0f + exp_of<FAST>(-g);
    return FAST ? __builtin_amdgcn_rcpf(e) : 1.0f / e;
}
// the normal distribution's cdf at g, given e = exp(-g^2 / 2)
template <bool FAST> __device__ __forceinline__ float cdf_of(float g, float e)
{
    if (!FAST) return 0.5f * erfcf(-g * 0.70710678118654752f);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.4f * 0.70710678118654752f, 1.0f));
    float q = 0.05026213f;
    q = fmaf(q, t, -0.18290149f);
    q = fmaf(q, t, 0.16908546f);
    q = fmaf(q, t, -0.00560756f);
    q = fmaf(q, t, 0.14143144f);
    q = fmaf(q, t, 0.16854198f);
    q = fmaf(q, t, 0.2078427f);
    q = fmaf(q, t, 0.2256696f);
    q = fmaf(q, t, 0.22567586f);
    const float half = 0.5f * t * q * e;                 // erfc(|x|) / 2
    return g < 0.0f ? half : 1.0f - half;
}
template <bool FAST> __device__ __forceinline__ float act_value(int act, float g)
{
    if (act == ACT_RELU) return g <= 0.0f ? 0.0f : g;
    if (act == ACT_GELU) return g * cdf_of<FAST>(g, FAST ? exp_of<FAST>(-0.5f * g * g) : 0.0f);
    const float s = sigmoid_of<FAST>(g);
    return act == ACT_SIGMOID ? s : g * s;
}
template <bool FAST> __device__ __forceinline__ void act_both(int act, float g, float &a, float &da)
{
    if (act == ACT_RELU) {
        a = g <= 0.0f ? 0.0f : g;
        da = g > 0.0f ? 1.0f : 0.0f;
    } else if (act == ACT_GELU) {
        const float e = exp_of<FAST>(-0.5f * g * g), cdf = cdf_of<FAST>(g, e);
        a = g * cdf;
        da = fmaf(g * e, 0.39894228040143268f, cdf);
    } else {
        // 1 - s of s within rounding of 1 has no digits left; exp(-g) s has all of them
        const float e = exp_of<FAST>(-g), s = FAST ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e), rest = g > 0.0f ? e * s : 1.0f - s;
        a = act == ACT_SIGMOID ? s : g * s;
        da = act == ACT_SIGMOID ? s * rest : s * (1.0f + g * rest);
    }
}

// ------------------------------------------------------------------ any sizes
// Products of float, on the float matrix cores (v_mfma_f32_32x32x2_f32, true float products), and of bf16 whose rows are no multiple
// of 16 bytes.  Operands pass through registers, 16 bytes in one access at any address (global memory needs no more
// alignment than an element's), a row's last ones one by one.  A block is 2 x 2 waves of 32 TM x 32 TN outputs; two tiles of the
// contracted dimension in LDS, the next one's loads in flight while this one's products run.

template <class T> __device__ __forceinline__ chunk16 load_chunk(const T *from)
{
    chunk16 c;
    __builtin_memcpy(&c, from, 16);
    return c;
}
// The first `left` elements, zeros behind them: the 16 bytes that end with them, moved down.  Element by element they would be a
// chain of loads for every chunk of a tile (forward, 1001 rows, 500->1333, us: 16.9 instead of 15.4).
template <class T> __device__ __forceinline__ chunk16 load_ending(const T *from, int left)
{
    constexpr int V = 16 / sizeof(T);
    const int drop = left < V ? V - left : 0;
    const chunk16 c = load_chunk(from - drop);
    uint64_t lo = (uint64_t)c[1] << 32 | c[0], hi = (uint64_t)c[3] << 32 | c[2];
    const int by = drop < V ? drop * (int)sizeof(T) * 8 : 128, bits = by % 64;
    if (by >= 64) lo = hi, hi = 0;
    if (bits) lo = lo >> bits | hi << (64 - bits), hi >>= bits;
    if (by == 128) lo = 0;
    return chunk16{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// ... of a row shorter than 16 bytes, in front of which there may be nothing
template <class T> __device__ __forceinline__ chunk16 load_short(const T *from, int left)
{
    constexpr int V = 16 / sizeof(T);
    T e[V];
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = j < left ? from[j] : T{};
    return __builtin_bit_cast(chunk16, e);
}

// All products of a wave's TM x TN tiles over the 32 bytes of K that its two halves hold 16 bytes of each
template <class T, int TM, int TN> __device__ __forceinline__ void multiply(f32x16 (&acc)[TM][TN], const chunk16 (&a)[TM], const chunk16 (&b)[TN])
{
#pragma unroll
    for (int k = 0; k < (sizeof(T) == 2 ? 1 : 4); ++k)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                if constexpr (sizeof(T) == 2) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_frag(a[i]), as_frag(b[j]), acc[i][j], 0, 0, 0);
                else acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i][k]), __uint_as_float(b[j][k]), acc[i][j], 0, 0, 0);
            }
}

enum { NT_FORWARD, NT_GRAD };
struct NtArgs {
    const void *a, *b;        // [M][K], [N][K] (forward: [2N][K])
    int M, N, K, k_per_split; // K split over blockIdx.y: part[split][M][N] (forward: [2N]) instead of the outputs
    float *part;
    const float *bias;        // forward
    float *P;                 // forward: both projections [M][2N]
    void *out;                // h [M][N], or dx [M][N]
    const void *old, *gate;   // gradient epilogue
    int act;
};

template <class T, int MODE, int TM, int TN>
__global__ __launch_bounds__(TPB) void k_gated_nt(NtArgs p)
{
    constexpr int V = 16 / sizeof(T), NQ = 4, CPR = 2 * NQ, DEPTH = CPR * V;      // of K a tile
    constexpr int PITCH = CPR * 16 + 16;           // bytes of a row: the reads of eight neighbouring rows lie on different banks
    constexpr int RA = 64 * TM, RB = 64 * TN, LA = RA * CPR / TPB, LB = RB * CPR / TPB, ROWS = TPB / CPR;
    constexpr bool FWD = MODE == NT_FORWARD;
    static_assert(!FWD || TN == 2, "a wave has gates and linear parts of 32 units");
    constexpr int WIDE = FWD ? RB / 2 : RB;        // outputs across
    __shared__ __align__(16) unsigned char lds[2][(RA + RB) * PITCH];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / 2, wn = wave % 2;
    const int across = (p.N + WIDE - 1) / WIDE, m0 = blockIdx.x / across * RA, n0 = blockIdx.x % across * WIDE;
    const int first = blockIdx.y * p.k_per_split, last = first + p.k_per_split < p.K ? first + p.k_per_split : p.K;
    // thread's chunks: column tid % CPR of rows tid / CPR + ROWS i
    const int c = tid % CPR * V, r0 = tid / CPR;
    const T *pa[LA], *pb[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int row = m0 + r0 + ROWS * i;
        pa[i] = (const T *)p.a + (size_t)(row < p.M ? row : p.M - 1) * p.K + c;      // nobody stores the rows behind the last
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int r = r0 + ROWS * i;               // forward: 32 units' gates, then the same units' linear parts, for each wave
        const int n = FWD ? n0 + r / 64 * 32 + r % 32 : n0 + r;
        const int unit = n < p.N ? n : p.N - 1;
        pb[i] = (const T *)p.b + (size_t)(FWD && r % 64 >= 32 ? p.N + unit : unit) * p.K + c;
    }
    chunk16 ca[LA], cb[LB];
    // only the last step of K ends inside a tile: splits are of whole ones
    auto load_all = [&](int k0, auto chunk) {
#pragma unroll
        for (int i = 0; i < LA; ++i) ca[i] = chunk(pa[i] + k0);
#pragma unroll
        for (int i = 0; i < LB; ++i) cb[i] = chunk(pb[i] + k0);
    };
    auto load = [&](int k0) {
        const int left = last - k0 - c;
        if (k0 + DEPTH <= last) load_all(k0, [](const T *from) { return load_chunk(from); });
        else if (p.K >= V) load_all(k0, [=](const T *from) { return load_ending(from, left); });
        else load_all(k0, [=](const T *from) { return load_short(from, left); });
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LA; ++i) *reinterpret_cast<chunk16 *>(&lds[buf][(r0 + ROWS * i) * PITCH + tid % CPR * 16]) = ca[i];
#pragma unroll
        for (int i = 0; i < LB; ++i) *reinterpret_cast<chunk16 *>(&lds[buf][(RA + r0 + ROWS * i) * PITCH + tid % CPR * 16]) = cb[i];
    };
    f32x16 acc[TM][TN] = {};
    const int steps = (last - first + DEPTH - 1) / DEPTH;
    load(first);
    store(0);
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
        if (s + 1 < steps) load(first + (s + 1) * DEPTH);
        const unsigned char *buf = lds[s & 1];
        chunk16 fa[2][TM], fb[2][TN];
        auto read = [&](int q) {
            const int at = (2 * q + lane / 32) * 16;
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[q & 1][i] = *reinterpret_cast<const chunk16 *>(buf + ((wm * TM + i) * 32 + lane % 32) * PITCH + at);
#pragma unroll
            for (int i = 0; i < TN; ++i) fb[q & 1][i] = *reinterpret_cast<const chunk16 *>(buf + (RA + (wn * TN + i) * 32 + lane % 32) * PITCH + at);
        };
        read(0);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (q + 1 < NQ) read(q + 1);
            __builtin_amdgcn_sched_barrier(0);       // the next reads ahead of the products that hide them
            multiply<T>(acc, fa[q & 1], fb[q & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (s + 1 < steps) store((s + 1) & 1);
    }
    // register r of lane l: row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = m0 + (wm * TM + i) * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
            if (row >= p.M) continue;
            if constexpr (FWD) {
                const int unit = n0 + wn * 32 + lane % 32;
                if (unit >= p.N) continue;
                float *P = (p.part ? p.part + (size_t)blockIdx.y * p.M * 2 * p.N : p.P) + (size_t)row * 2 * p.N + unit;
                const float g = acc[i][0][r] + (!p.part && p.bias ? p.bias[unit] : 0.0f), u = acc[i][1][r] + (!p.part && p.bias ? p.bias[p.N + unit] : 0.0f);
                P[0] = g;
                P[p.N] = u;
                if (!p.part) ((T *)p.out)[(size_t)row * p.N + unit] = from_f32<T>(act_value<kFast<T>>(p.act, g) * u);
            } else {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int col = n0 + (wn * TN + j) * 32 + lane % 32;
                    if (col >= p.N) continue;
                    const size_t at = (size_t)row * p.N + col;
                    const T *old = (const T *)p.old, *gate = (const T *)p.gate;
                    if (p.part) p.part[(size_t)blockIdx.y * p.M * p.N + at] = acc[i][j][r];
                    else
                        ((T *)p.out)[at] = grad_out<T>(acc[i][j][r], old != nullptr, old ? old[at] : from_f32<T>(0.0f), gate != nullptr,
                                                       gate ? gate[at] : from_f32<T>(0.0f));
                }
            }
        }
}

// dw[M][N] += a^T b with a [rows][M], b [rows][N], and (where db is not NULL) db[M] += the columns' sums of a, over the rows of split
// blockIdx.y; with several splits part[split][M][N] and, behind all of it, [split][M] = their sums.
// A step is 64 rows of bf16 (of 32, whose loads the products do not cover, dw of 4006 x 1001 from 8192 rows took 121 us instead of 106), read
// across the rows by transposing reads (tr_frag), or 32 of float.  The first blocks of a row of tiles sum a's columns as they pass
// (a pass of its own over a of 1024 x 4096 floats: 9 us).
template <class T, int TM, int TN>
__global__ __launch_bounds__(TPB) void k_gated_tn(const T *__restrict__ a, const T *__restrict__ b, int rows, int M, int N, int rows_per_split,
                                                  float *dw, float *db, float *part)
{
    constexpr int V = 16 / sizeof(T), DEPTH = 128 / sizeof(T), CA = 64 * TM, CB = 64 * TN;
    constexpr int LA = DEPTH * CA / V / TPB, LB = DEPTH * CB / V / TPB;
    static_assert(LA >= 1 && LB >= 1, "a chunk for every thread");
    static_assert(TPB % (CA / V) == 0, "a thread's chunks of a have the same columns");
    __shared__ __align__(16) T lds[2][DEPTH * (CA + CB)];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / 2, wn = wave % 2;
    const int across = (N + CB - 1) / CB, m0 = blockIdx.x / across * CA, n0 = blockIdx.x % across * CB;
    const int first = blockIdx.y * rows_per_split, last = first + rows_per_split < rows ? first + rows_per_split : rows;
    chunk16 ca[LA], cb[LB];
    // Columns behind the last are never stored, so that a row's last 16 bytes may go on into the rows behind it, where there are some.
    // One test for all of a step's loads: with one for each they waited for one another (dw of 4006 x 1001 from 8192 rows 210 us)
    auto load_all = [&](int at, auto chunk) {
        auto fetch = [&](auto &to, const T *from, int width, int c0, auto columns) {
            constexpr int CPR = decltype(columns)::value / V;
#pragma unroll
            for (int i = 0; i < (int)(sizeof(to) / sizeof(to[0])); ++i) {
                const int id = tid + TPB * i;
                to[i] = chunk(from, width, at + id / CPR, c0 + id % CPR * V);
            }
        };
        fetch(ca, a, M, m0, std::integral_constant<int, CA>{});
        fetch(cb, b, N, n0, std::integral_constant<int, CB>{});
    };
    const int narrow = M < N ? M : N;
    auto load = [&](int at) {
        if (at + DEPTH <= last && (size_t)(rows - at - DEPTH) * narrow >= V)
            load_all(at, [](const T *from, int width, int r, int c) { return load_chunk(from + (size_t)r * width + (c < width ? c : 0)); });
        else if (narrow >= V)
            load_all(at, [=](const T *from, int width, int r, int c) {
                const chunk16 v = load_ending(from + (size_t)(r < last ? r : last - 1) * width + c, width - c);
                return r < last ? v : chunk16{0u, 0u, 0u, 0u};
            });
        else
            load_all(at, [=](const T *from, int width, int r, int c) { return load_short(from + (size_t)r * width + c, r < last ? width - c : 0); });
    };
    auto put = [&](T *tile, auto &from, auto columns) {
        constexpr int C = decltype(columns)::value, CPR = C / V;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(from) / sizeof(from[0])); ++i) {
            const int id = tid + TPB * i, r = id / CPR, c = id % CPR;
            const int slot = sizeof(T) == 2 ? ((((c >> 1) ^ wg_swz<C>(r)) << 1) | (c & 1)) : c;
            *reinterpret_cast<chunk16 *>(tile + r * C + slot * V) = from[i];
        }
    };
    float column[V] = {};
    const bool sums = db && n0 == 0;
    auto store = [&](int buf) {
        if (sums)
#pragma unroll
            for (int i = 0; i < LA; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) column[j] += chunk_value<T>(ca[i], j);
        put(lds[buf], ca, std::integral_constant<int, CA>{});
        put(lds[buf] + DEPTH * CA, cb, std::integral_constant<int, CB>{});
    };
    f32x16 acc[TM][TN] = {};
    const int steps = (last - first + DEPTH - 1) / DEPTH;
    load(first);
    store(0);
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
        if (s + 1 < steps) load(first + (s + 1) * DEPTH);
        const T *ta = lds[s & 1], *tb = ta + DEPTH * CA;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int q = 0; q < DEPTH / 16; ++q) {
                bf16x8_t fa[TM], fb[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[i] = tr_frag<CA>((const uint16_t *)ta, (wm * TM + i) * 32, q * 16, lane);
#pragma unroll
                for (int i = 0; i < TN; ++i) fb[i] = tr_frag<CB>((const uint16_t *)tb, (wn * TN + i) * 32, q * 16, lane);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
            }
        } else {
            constexpr int AHEAD = 4;                     // rows' pairs read before the products that need them
            float fa[2][AHEAD][TM], fb[2][AHEAD][TN];
            auto read = [&](int h) {
#pragma unroll
                for (int q = 0; q < AHEAD; ++q) {
                    const int k = (h * AHEAD + q) * 2 + lane / 32;
#pragma unroll
                    for (int i = 0; i < TM; ++i) fa[h & 1][q][i] = ta[k * CA + (wm * TM + i) * 32 + lane % 32];
#pragma unroll
                    for (int i = 0; i < TN; ++i) fb[h & 1][q][i] = tb[k * CB + (wn * TN + i) * 32 + lane % 32];
                }
            };
            read(0);
#pragma unroll
            for (int h = 0; h < DEPTH / 2 / AHEAD; ++h) {
                if (h + 1 < DEPTH / 2 / AHEAD) read(h + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[h & 1][q][i], fb[h & 1][q][j], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (s + 1 < steps) store((s + 1) & 1);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = m0 + (wm * TM + i) * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
            if (row >= M) continue;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int col = n0 + (wn * TN + j) * 32 + lane % 32;
                if (col >= N) continue;
                if (part) part[((size_t)blockIdx.y * M + row) * N + col] = acc[i][j][r];
                else dw[(size_t)row * N + col] += acc[i][j][r];
            }
        }
    if (!sums) return;
    __syncthreads();
    float *meet = reinterpret_cast<float *>(lds[0]);       // [TPB / (CA / V)][CA]
#pragma unroll
    for (int j = 0; j < V; ++j) meet[tid * V + j] = column[j];
    __syncthreads();
    if (tid >= CA || m0 + tid >= M) return;
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < TPB / (CA / V); ++r) sum += meet[r * CA + tid];
    if (part) part[(size_t)gridDim.y * M * N + (size_t)blockIdx.y * M + m0 + tid] = sum;
    else db[m0 + tid] += sum;
}

// dw[n] += the sums of all splits part[split][n], in their order, and where db is not NULL db[m] += those of the [split][m] behind them; n and
// m multiples of V
template <int V>
__global__ __launch_bounds__(TPB) void k_gated_tn_join(const float *__restrict__ part, int splits, size_t n, float *dw, size_t m, float *db)
{
    size_t i = ((size_t)blockIdx.x * TPB + threadIdx.x) * V;
    if (i >= n) {
        i -= n;
        if (!db || i >= m) return;
        part += splits * n;
        n = m;
        dw = db;
    }
    typedef vec_t<float, V> vec;
    vec sum = {};
    for (int k = 0; k < splits; ++k) {
        const vec v = *reinterpret_cast<const vec *>(part + (size_t)k * n + i);
#pragma unroll
        for (int j = 0; j < V; ++j) sum.e[j] += v.e[j];
    }
    vec d = *reinterpret_cast<vec *>(dw + i);
#pragma unroll
    for (int j = 0; j < V; ++j) d.e[j] += sum.e[j];
    *reinterpret_cast<vec *>(dw + i) = d;
}

// dx from the sums of all splits, part[split][n]
template <class T>
__global__ __launch_bounds__(TPB) void k_gated_grad_join(const float *__restrict__ part, int splits, size_t n, T *out, const T *old, const T *gate)
{
    const size_t i = (size_t)blockIdx.x * TPB + threadIdx.x;
    if (i >= n) return;
    float sum = 0.0f;
    for (int k = 0; k < splits; ++k) sum += part[(size_t)k * n + i];
    out[i] = grad_out<T>(sum, old != nullptr, old ? old[i] : from_f32<T>(0.0f), gate != nullptr, gate ? gate[i] : from_f32<T>(0.0f));
}

// Projections of V units from the sums of a product whose K was in `splits` parts, part[split][rows][2F]; F a multiple of V, h aligned
// to V elements
template <class T, int V>
__global__ __launch_bounds__(TPB) void k_gated_join(const float *__restrict__ part, int splits, const float *__restrict__ bias, float *__restrict__ P,
                                                    T *__restrict__ h, int rows, int F, int act)
{
    typedef vec_t<float, V> vecf;
    const size_t i = ((size_t)blockIdx.x * TPB + threadIdx.x) * V, n = (size_t)rows * F;
    if (i >= n) return;
    const size_t row = i / F, at = row * 2 * F + (i - row * F);
    const int unit = (int)(i - row * F);
    vecf g = {}, u = {};
    auto add = [](vecf &t, const float *from) {
        const vecf v = *reinterpret_cast<const vecf *>(from);
#pragma unroll
        for (int j = 0; j < V; ++j) t.e[j] += v.e[j];
    };
    for (int k = 0; k < splits; ++k) {
        add(g, part + (size_t)k * 2 * n + at);
        add(u, part + (size_t)k * 2 * n + at + F);
    }
    if (bias) {
        add(g, bias + unit);
        add(u, bias + F + unit);
    }
    *reinterpret_cast<vecf *>(P + at) = g;
    *reinterpret_cast<vecf *>(P + at + F) = u;
    vec_t<T, V> v;
#pragma unroll
    for (int j = 0; j < V; ++j) v.e[j] = from_f32<T>(act_value<kFast<T>>(act, g.e[j]) * u.e[j]);
    *reinterpret_cast<vec_t<T, V> *>(h + i) = v;
}

// D from dh and the projections, V units a thread (F a multiple of V, dh aligned to V elements).  dh_parts: instead of dh its `parts`
// float sums [parts][n].  rest: NULL, or what rounding takes from D
template <class T, int V>
__global__ __launch_bounds__(TPB) void k_gated_grad(const T *__restrict__ dh, const float *__restrict__ dh_parts, int parts, const float *__restrict__ P,
                                                    T *__restrict__ D, T *__restrict__ rest, size_t n, int F, int act)
{
    const size_t i = ((size_t)blockIdx.x * TPB + threadIdx.x) * V;
    if (i >= n) return;
    const size_t row = i / F, at = row * 2 * F + (i - row * F);
    typedef vec_t<T, V> vec;
    typedef vec_t<float, V> vecf;
    float d[V] = {};
    if (dh_parts) {
        for (int k = 0; k < parts; ++k) {
            const vecf v = *reinterpret_cast<const vecf *>(dh_parts + (size_t)k * n + i);
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] += v.e[j];
        }
    } else {
        const vec v = *reinterpret_cast<const vec *>(dh + i);
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = to_f32(v.e[j]);
    }
    const vecf g = *reinterpret_cast<const vecf *>(P + at), u = *reinterpret_cast<const vecf *>(P + at + F);
    vec dg, du, rg, ru;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float a, da;
        act_both<kFast<T>>(act, g.e[j], a, da);
        const float vg = d[j] * u.e[j] * da, vu = d[j] * a;
        dg.e[j] = from_f32<T>(vg);
        du.e[j] = from_f32<T>(vu);
        rg.e[j] = from_f32<T>(rounding_took(vg, to_f32(dg.e[j])));
        ru.e[j] = from_f32<T>(rounding_took(vu, to_f32(du.e[j])));
    }
    *reinterpret_cast<vec *>(D + at) = dg;
    *reinterpret_cast<vec *>(D + at + F) = du;
    if (!rest) return;
    *reinterpret_cast<vec *>(rest + at) = rg;
    *reinterpret_cast<vec *>(rest + at + F) = ru;
}

// ------------------------------------------------------------------ many rows of whole 16 bytes
// One kernel for three products of rows with rows, x [rows][K] and w [.][K]:
//   MM_FORWARD  both projections, activation and product.  A block's weights are the gates and the linear parts of BU units, a wave's
//               those of the same units in the same lanes, so that the activation meets both in registers
//   MM_PROJECT  dh of a 1x1 convolution's input gradient, w its transposed filter [F][K], turned into D from the projections at once:
//               dh is neither stored nor rounded
//   MM_DX       dx = D W of a float layer (of a bf16 one it is the gather kernel's)
// A block takes BP rows and 2 BU weight rows, a wave BP / WP of BU / WU units (MM_FORWARD) or twice as many columns.
// Tiles of 128 bytes of K come HBM / L2 -> LDS without passing registers into a ring of two (see mfma_common.h; the swizzle of a tile's
// 16-byte chunks is applied by choosing which one a lane fetches).  Fragments are read one step of 32 bytes ahead of the products that
// need them; the barrier that publishes the next tile lies before a tile's last products, when every wave has all of the tile in registers, and
// the slot is filled again at once.
// 8192 rows, 4096->11008 of bf16, us (1478 GFLOP), launched by itself time after time: MM_FORWARD 1310, 721 MB of projections and 180 of h among them, the
// gather kernel alone on as large a product 1316.  Between the other kernels of a mini-batch it takes 1440 to 1452.
// `rest`: x is the sum of two tensors; K is walked twice with the same weights.
enum { MM_FORWARD, MM_PROJECT, MM_DX };
struct MmArgs {
    const void *x, *rest, *w;        // [rows][K], [2F or N][K]
    int rows, K, N;                  // N: units or columns
    const float *bias;
    float *P;                        // [rows][2N], written or (MM_PROJECT) read
    void *out;                       // h [rows][N], D [rows][2N], dx [rows][N]
    const void *old, *gate;          // MM_DX: see grad_out()
    unsigned x_bytes, w_bytes;
    int tiles_p, tiles_u, act;
    void *out_rest = nullptr;        // MM_PROJECT: what rounding takes from D, or NULL
};

// Rows of tiles that go together: the 32 blocks that an XCD's units run at a time are then 4 x 8 tiles and ask the L2 for 12 operand tiles, in
// one row of tiles for 33.  MM_FORWARD at the size above, us, with 2, 4, 8 and 16 rows together: 1358, 1327, 1343, 1460; with 4 and the
// projections stored past the L2 1310.
constexpr int MM_ROWS = 4;

template <class T, int MODE, int BP, int BU, int WP, int WU>
__global__ __launch_bounds__(WP *WU * 64, 2) void k_gated_mfma(MmArgs p)
{
    constexpr bool FWD = MODE == MM_FORWARD;
    constexpr int ES = sizeof(T), NW = WP * WU, BKB = 128, BC = 2 * BU, STAGE = (BP + BC) * BKB;      // bytes
    constexpr int XL = BP / (8 * NW), WL = BC / (8 * NW);       // wave-wide loads a tile, 8 rows each
    constexpr int TP = BP / WP / 32, TC = 2 * BU / WU / 32, TU = TC / 2, KSUB = BKB / 32;
    static_assert(XL >= 1 && WL >= 1 && TP >= 1 && TU >= 1, "tile and waves");
    extern __shared__ __align__(16) unsigned char smem[];
    const lds_addr_of lds_of(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave % WP, wu = wave / WP;
    auto swz = [](int row) { return (row >> 1) & 7; };
    const int lrow = lane / 8, lc = (lane % 8) ^ swz(wave * 8 + lrow);      // the same for every load: they lie 8 NW rows apart

    constexpr int WIDE = FWD ? BU : BC;
    const int bid = xcd_remap(blockIdx.x, gridDim.x);
    const int per = MM_ROWS * p.tiles_u, first = bid / per * MM_ROWS, here = p.tiles_p - first < MM_ROWS ? p.tiles_p - first : MM_ROWS;
    const int row0 = (first + bid % per % here) * BP, col0 = bid % per / here * WIDE;

    constexpr unsigned OOB = 0x80000000u;
    __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p.x), 0, (int)p.x_bytes, 0x00020000);
    __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p.w), 0, (int)p.w_bytes, 0x00020000);
    // rows past the end lie behind the buffer and read zeros; gates past the last unit read linear parts, whose products nobody stores
    const unsigned pitch = (unsigned)p.K * ES;
    unsigned xoff[XL], woff[WL];
#pragma unroll
    for (int i = 0; i < XL; ++i) xoff[i] = (unsigned)(row0 + (i * NW + wave) * 8 + lrow) * pitch + 16u * lc;
#pragma unroll
    for (int i = 0; i < WL; ++i) {
        const int r = (i * NW + wave) * 8 + lrow, row = !FWD || r < BU ? col0 + r : p.N + col0 + r - BU;
        woff[i] = (unsigned)row * pitch + 16u * lc;
    }
    const int KT = (int)((pitch + BKB - 1) / BKB), n_it = p.rest ? 2 * KT : KT;
    int at = 0;                              // next tile to ask for
    auto issue = [&](int slot) {
        unsigned char *sw = smem + slot * STAGE, *sx = sw + BC * BKB;
        if (at == KT && p.rest) xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p.rest), 0, (int)p.x_bytes, 0x00020000);
        const unsigned ko = (unsigned)(at < KT ? at : at - KT) * BKB;
        const bool in = at < n_it && ko + 16u * lc < pitch;
#pragma unroll
        for (int i = 0; i < XL; ++i) dma16(xr, lds_of(sx + (i * NW + wave) * 8 * BKB), in ? xoff[i] + ko : OOB);
#pragma unroll
        for (int i = 0; i < WL; ++i) dma16(wr, lds_of(sw + (i * NW + wave) * 8 * BKB), in ? woff[i] + ko : OOB);
        ++at;
    };
    f32x16 acc[TP][TC];
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int b = 0; b < TC; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    const int frow = lane & 31, fhalf = lane >> 5;
    // column of a wave's tile b inside the block's weight rows
    auto tile_row = [&](int b) { return FWD ? b / TU * BU + (wu * TU + b % TU) * 32 : (wu * TC + b) * 32; };
    auto load_frags = [&](int slot, int k, chunk16(&fx)[TP], chunk16(&fw)[TC]) {
        const unsigned char *cw = smem + slot * STAGE, *cx = cw + BC * BKB;
        const int ch = 2 * k + fhalf;
#pragma unroll
        for (int b = 0; b < TC; ++b) {
            const int row = tile_row(b) + frow;
            fw[b] = *reinterpret_cast<const chunk16 *>(cw + row * BKB + ((ch ^ swz(row)) << 4));
        }
#pragma unroll
        for (int a = 0; a < TP; ++a) {
            const int row = (wp * TP + a) * 32 + frow;
            fx[a] = *reinterpret_cast<const chunk16 *>(cx + row * BKB + ((ch ^ swz(row)) << 4));
        }
    };
    issue(0);
    issue(1);
    WAIT_VMCNT(XL + WL);
    WAIT_LGKMCNT(0);
    __builtin_amdgcn_s_barrier();
    chunk16 fx[2][TP], fw[2][TC];
    load_frags(0, 0, fx[0], fw[0]);
    for (int it = 0; it < n_it; ++it) {
        const int slot = it & 1;
#pragma unroll
        for (int j = 0; j + 1 < KSUB; ++j) {
            load_frags(slot, j + 1, fx[(j + 1) & 1], fw[(j + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);               // keep the reads ahead of the products that hide them
            multiply<T>(acc, fx[j & 1], fw[j & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        WAIT_LGKMCNT(0);                                     // this wave has read all of the tile
        WAIT_VMCNT(0);                                       // its share of the next one has landed
        __builtin_amdgcn_s_barrier();
        load_frags(slot ^ 1, 0, fx[0], fw[0]);
        __builtin_amdgcn_sched_barrier(0);
        issue(slot);
        multiply<T>(acc, fx[1], fw[1]);
        __builtin_amdgcn_sched_barrier(0);
    }
    WAIT_VMCNT(0);
    // register r of lane l: row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32
    auto row_of = [&](int a, int r) { return row0 + (wp * TP + a) * 32 + 8 * (r / 4) + 4 * fhalf + r % 4; };
    if constexpr (FWD) {
#pragma unroll
        for (int b = 0; b < TU; ++b) {
            const int unit = col0 + tile_row(b) + frow;
            if (unit >= p.N) continue;
            const float bg = p.bias ? p.bias[unit] : 0.0f, bu = p.bias ? p.bias[p.N + unit] : 0.0f;
#pragma unroll
            for (int a = 0; a < TP; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = row_of(a, r);
                    if (row >= p.rows) continue;
                    const float g = acc[a][b][r] + bg, u = acc[a][TU + b][r] + bu;
                    float *P = p.P + (size_t)row * 2 * p.N + unit;          // read again by the backward pass: not through the L2
                    __builtin_nontemporal_store(g, P);
                    __builtin_nontemporal_store(u, P + p.N);
                    ((T *)p.out)[(size_t)row * p.N + unit] = from_f32<T>(act_value<kFast<T>>(p.act, g) * u);
                }
        }
    } else {
#pragma unroll
        for (int b = 0; b < TC; ++b) {
            const int col = col0 + tile_row(b) + frow;
            if (col >= p.N) continue;
#pragma unroll
            for (int a = 0; a < TP; ++a) {
                if constexpr (MODE == MM_PROJECT) {
                    float g[16], u[16];                      // asked for together
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int row = row_of(a, r);
                        const float *P = p.P + (size_t)(row < p.rows ? row : p.rows - 1) * 2 * p.N + col;
                        g[r] = P[0];
                        u[r] = P[p.N];
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int row = row_of(a, r);
                        float v, dv;
                        act_both<kFast<T>>(p.act, g[r], v, dv);
                        if (row >= p.rows) continue;
                        T *D = (T *)p.out + (size_t)row * 2 * p.N + col;
                        const float dg = acc[a][b][r] * u[r] * dv, du = acc[a][b][r] * v;
                        D[0] = from_f32<T>(dg);
                        D[p.N] = from_f32<T>(du);
                        if (!p.out_rest) continue;
                        T *rest = (T *)p.out_rest + (size_t)row * 2 * p.N + col;
                        rest[0] = from_f32<T>(rounding_took(dg, round_to<T>(dg)));
                        rest[p.N] = from_f32<T>(rounding_took(du, round_to<T>(du)));
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int row = row_of(a, r);
                        if (row >= p.rows) continue;
                        const size_t i = (size_t)row * p.N + col;
                        const T *old = (const T *)p.old, *gate = (const T *)p.gate;
                        ((T *)p.out)[i] = grad_out<T>(acc[a][b][r], old != nullptr, old ? old[i] : from_f32<T>(0.0f), gate != nullptr,
                                                      gate ? gate[i] : from_f32<T>(0.0f));
                    }
                }
            }
        }
    }
}

// How a product of any sizes is cut: into tiles of 128 x 128, or of 64 rows, and the contracted dimension into splits of 256 at the
// least.  The units take their blocks in step, so what counts is the fullest unit's share of the products: `each` outputs a block, for a
// lone block, whose barriers nobody fills, half as many again, and for splits their sums written and read (a float's 8 bytes
// against products at about 30 a byte).
struct AnyPlan {
    bool small;
    int splits, per_split;
};
AnyPlan any_plan(long long rows, long long across, int tile_across, int small_across, int K, int sums)
{
    AnyPlan best{};
    double least = 1e300;
    for (const bool small : {false, true}) {
        const int r = small ? 64 : 128, c = small ? small_across : tile_across;
        const long long tiles = ((rows + r - 1) / r) * ((across + c - 1) / c);
        for (long long splits = 1; splits <= (K + 255) / 256 && (splits == 1 || tiles * splits <= 1024); ++splits) {
            const int per = (int)(((K + splits - 1) / splits + 63) / 64 * 64);
            const long long full = (tiles * ((K + per - 1) / per) + 255) / 256;
            const double cost = (double)(full == 1 ? 1.5 : full) * r * c * sums * (small ? 1.15 : 1.0) * per +
                                (splits > 1 ? (double)rows * across * sums * splits * 8 * 30 / 256 : 0.0);
            if (cost < least) {
                least = cost;
                best = {small, (K + per - 1) / per, per};
            }
        }
    }
    return best;
}
AnyPlan forward_plan(int rows, int C, int F) { return any_plan(rows, F, 64, 64, C, 2); }
AnyPlan dgrad_plan(int rows, int C, int F) { return any_plan(rows, C, 128, 64, 2 * F, 1); }
AnyPlan wgrad_plan(int rows, int C, int F) { return any_plan(2ll * F, C, 128, 64, rows, 1); }

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

template <class T, int MODE, int BP, int BU, int WP, int WU>
static hipError_t launch_mm_tile(MmArgs a, hipStream_t s)
{
    constexpr int bytes = 2 * (BP + 2 * BU) * 128, wide = MODE == MM_FORWARD ? BU : 2 * BU;
    auto kernel = k_gated_mfma<T, MODE, BP, BU, WP, WU>;
    if (bytes > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    a.tiles_p = (a.rows + BP - 1) / BP;
    a.tiles_u = (a.N + wide - 1) / wide;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.tiles_p * a.tiles_u), dim3(WP * WU * 64), bytes, s, a);
    return hipGetLastError();
}

// tiles of a product, counted in weight rows
static long long mm_tiles(int rows, long long weight_rows, int tile_p, int tile_w) { return (rows + tile_p - 1) / tile_p * ((weight_rows + tile_w - 1) / tile_w); }

// The tile whose rounds of the chip are the least work: a block of 256 x 256 or 256 x 128 to a unit, or two of 128 x 128, whose products
// take 1.05 and 1.15 times as long each (4096 rows, 2048->5632, us, by itself: 704 of the first, three rounds, 204; 2816 of the last, six, 234; the first
// between the other kernels of a mini-batch 226 to 229)
template <class T, int MODE> static hipError_t launch_mm(MmArgs a, hipStream_t s)
{
    const long long w = MODE == MM_FORWARD ? 2ll * a.N : a.N;
    auto rounds = [&](int tile_p, int tile_w, int slots) { return (double)((mm_tiles(a.rows, w, tile_p, tile_w) + slots - 1) / slots); };
    const double whole = rounds(256, 256, 256) * 4.0, half = rounds(256, 128, 256) * 2.0 * 1.05, small = rounds(128, 128, 512) * 2.0 * 1.15;
    if (whole <= half && whole <= small) return launch_mm_tile<T, MODE, 256, 128, 2, 4>(a, s);
    if (half <= small) return launch_mm_tile<T, MODE, 256, 64, 4, 2>(a, s);
    return launch_mm_tile<T, MODE, 128, 64, 2, 2>(a, s);
}

// Whether k_gated_mfma takes a product: rows of whole 16 bytes, offsets that 32 bits hold, those of a tile's rows behind the last ones among
// them, and tiles enough for it.  Of few the other kernels split K (forward, us, this / those: bf16, 1024 rows, 1024->1024, 128 tiles, 18.9 / 16.8,
// 2048 rows, 512->1024, 256 tiles, 16.4 / 23.6; float, 2048 rows, 512->1024, 256 tiles, 45.6 / 43.7).
static bool mm_takes(int dt, int rows, int K, long long weight_rows)
{
    const size_t es = dt_size(dt);
    return K * es % 16 == 0 && K * es <= 2u << 20 && (size_t)rows * K * es < (1u << 31) && (size_t)weight_rows * K * es < (1u << 31) && rows > 64 &&
           mm_tiles(rows, weight_rows, 128, 128) >= (dt == DT_F32 ? 512 : 192);
}

size_t gated_workspace(int dt, int rows, int C, int F, bool rest, bool parts)
{
    const size_t walks = rest ? 2 : 1;
    if (gated_mfma(dt, rows, C, F)) return mm_takes(dt, rows, C, 2ll * F) ? 0 : walks * conv_gather_mfma_raw_workspace(rows_product(rows, C, 2 * F, false));
    auto sums = [](size_t splits, size_t n) { return splits > 1 ? splits * n * sizeof(float) : 0; };
    size_t most = sums(wgrad_plan(rows, C, F).splits, (size_t)2 * F * (C + 1));
    const size_t forward = mm_takes(dt, rows, C, 2ll * F) ? 0 : sums(forward_plan(rows, C, F).splits * walks, (size_t)rows * 2 * F);
    const size_t dgrad = parts || (dt == DT_F32 && mm_takes(dt, rows, 2 * F, C)) ? 0 : sums(dgrad_plan(rows, C, F).splits, (size_t)rows * C);
    for (const size_t v : {forward, dgrad}) most = v > most ? v : most;
    return most;
}

#define GATED_T(dt, ...)                                              \
    do {                                                              \
        if ((dt) == DT_F32) { using T = float; __VA_ARGS__; }         \
        else { using T = bf16_t; __VA_ARGS__; }                       \
    } while (0)

static hipError_t join(int dt, int act, const float *part, int splits, const float *bias, float *P, void *h, int rows, int F, hipStream_t s)
{
    const size_t n = (size_t)rows * F;
    const bool four = F % 4 == 0 && (uintptr_t)h % (4 * dt_size(dt)) == 0;       // the caller's h may lie anywhere
    const dim3 grid((unsigned)((n / (four ? 4 : 1) + TPB - 1) / TPB));
    if (four) GATED_T(dt, hipLaunchKernelGGL((k_gated_join<T, 4>), grid, dim3(TPB), 0, s, part, splits, bias, P, (T *)h, rows, F, act));
    else GATED_T(dt, hipLaunchKernelGGL((k_gated_join<T, 1>), grid, dim3(TPB), 0, s, part, splits, bias, P, (T *)h, rows, F, act));
    return hipGetLastError();
}

hipError_t gated_fwd(int dt, int act, const void *x, const void *rest, const void *w, const float *bias, float *P, void *h, int rows, int C, int F, bool panels,
                     void *workspace, hipStream_t s)
{
    if (mm_takes(dt, rows, C, 2ll * F)) {
        if (panels) return hipErrorInvalidValue;
        const size_t es = dt_size(dt);
        MmArgs a{x, rest, w, rows, C, F, bias, P, h, nullptr, nullptr, (unsigned)((size_t)rows * C * es), (unsigned)((size_t)2 * F * C * es), 0, 0, act};
        return dt == DT_F32 ? launch_mm<float, MM_FORWARD>(a, s) : launch_mm<bf16_t, MM_FORWARD>(a, s);
    }
    if (gated_mfma(dt, rows, C, F)) {
        int splits = 0, more = 0;
        const GatherConv g = rows_product(rows, C, 2 * F, panels);
        hipError_t e = conv_gather_mfma_raw(x, w, g, (float *)workspace, &splits, s);
        if (e == hipSuccess && rest) e = conv_gather_mfma_raw(rest, w, g, (float *)workspace + (size_t)splits * rows * 2 * F, &more, s);
        if (e != hipSuccess) return e;
        splits += more;
        return join(dt, act, (const float *)workspace, splits, bias, P, h, rows, F, s);
    }
    if (panels) return hipErrorInvalidValue;
    const AnyPlan p = forward_plan(rows, C, F);
    const int splits = p.splits * (rest ? 2 : 1);
    const dim3 grid((unsigned)((F + 63) / 64) * ((rows + (p.small ? 63 : 127)) / (p.small ? 64 : 128)), p.splits);
    for (int walk = 0; walk * p.splits < splits; ++walk) {
        float *part = splits > 1 ? (float *)workspace + (size_t)walk * p.splits * rows * 2 * F : nullptr;
        NtArgs a{walk ? rest : x, w, rows, F, C, p.per_split, part, bias, P, h, nullptr, nullptr, act};
        if (p.small) GATED_T(dt, hipLaunchKernelGGL((k_gated_nt<T, NT_FORWARD, 1, 2>), grid, dim3(TPB), 0, s, a));
        else GATED_T(dt, hipLaunchKernelGGL((k_gated_nt<T, NT_FORWARD, 2, 2>), grid, dim3(TPB), 0, s, a));
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || splits == 1 ? e : join(dt, act, (const float *)workspace, splits, bias, P, h, rows, F, s);
}

hipError_t gated_grad(int dt, int act, const void *dh, int dh_parts, const float *P, void *D, void *rest, int rows, int F, hipStream_t s)
{
    const float *parts = dh_parts ? (const float *)dh : nullptr;
    const size_t n = (size_t)rows * F;
    const bool four = F % 4 == 0 && (parts || (uintptr_t)dh % (4 * dt_size(dt)) == 0);      // the caller's dh may lie anywhere
    const dim3 grid((unsigned)((n / (four ? 4 : 1) + TPB - 1) / TPB));
    if (four) GATED_T(dt, hipLaunchKernelGGL((k_gated_grad<T, 4>), grid, dim3(TPB), 0, s, (const T *)dh, parts, dh_parts, P, (T *)D, (T *)rest, n, F, act));
    else GATED_T(dt, hipLaunchKernelGGL((k_gated_grad<T, 1>), grid, dim3(TPB), 0, s, (const T *)dh, parts, dh_parts, P, (T *)D, (T *)rest, n, F, act));
    return hipGetLastError();
}

bool gated_projects(int rows, int K, int F) { return F % 8 == 0 && mm_takes(DT_BF16, rows, K, F); }

hipError_t gated_project(int act, const void *dz, const void *wt, bool panels, const float *P, void *D, void *rest, int rows, int K, int F, hipStream_t s)
{
    if (panels || !gated_projects(rows, K, F)) return hipErrorInvalidValue;
    MmArgs a{dz, nullptr, wt, rows, K, F, nullptr, const_cast<float *>(P), D, nullptr, nullptr, (unsigned)((size_t)rows * K * 2),
             (unsigned)((size_t)F * K * 2), 0, 0, act, rest};
    return launch_mm<bf16_t, MM_PROJECT>(a, s);
}

int gated_dgrad_parts(int rows, int C, int F) { return dgrad_plan(rows, C, F).splits; }

hipError_t gated_dgrad_direct(int dt, const void *D, const void *wt, void *dx, bool parts, GradEpi epi, int rows, int C, int F, void *workspace,
                              hipStream_t s)
{
    const void *old = epi.accum ? (epi.accum_from ? epi.accum_from : dx) : nullptr;
    if (!parts && dt == DT_F32 && mm_takes(dt, rows, 2 * F, C)) {
        MmArgs a{D, nullptr, wt, rows, 2 * F, C, nullptr, nullptr, dx, old, epi.gate, (unsigned)((size_t)rows * 2 * F * 4), (unsigned)((size_t)2 * F * C * 4), 0, 0, 0};
        return launch_mm<float, MM_DX>(a, s);
    }
    const AnyPlan p = dgrad_plan(rows, C, F);
    NtArgs a{D, wt, rows, C, 2 * F, p.per_split, parts ? (float *)dx : p.splits > 1 ? (float *)workspace : nullptr, nullptr, nullptr, dx, old, epi.gate, 0};
    const int tile = p.small ? 64 : 128;
    const dim3 grid((unsigned)((C + tile - 1) / tile) * ((rows + tile - 1) / tile), p.splits);
    if (p.small) GATED_T(dt, hipLaunchKernelGGL((k_gated_nt<T, NT_GRAD, 1, 1>), grid, dim3(TPB), 0, s, a));
    else GATED_T(dt, hipLaunchKernelGGL((k_gated_nt<T, NT_GRAD, 2, 2>), grid, dim3(TPB), 0, s, a));
    if (p.splits > 1 && !parts) {
        const size_t n = (size_t)rows * C;
        GATED_T(dt, hipLaunchKernelGGL((k_gated_grad_join<T>), dim3((unsigned)((n + TPB - 1) / TPB)), dim3(TPB), 0, s, (const float *)workspace, p.splits, n,
                                       (T *)dx, (const T *)old, (const T *)epi.gate));
    }
    return hipGetLastError();
}

hipError_t gated_wgrad_direct(int dt, const void *x, const void *D, float *dw, float *db, int rows, int C, int F, void *workspace, hipStream_t s)
{
    const int M = 2 * F;
    const AnyPlan p = wgrad_plan(rows, C, F);
    float *part = p.splits > 1 ? (float *)workspace : nullptr;
    const int tile = p.small ? 64 : 128;
    const dim3 grid((unsigned)((C + tile - 1) / tile) * ((M + tile - 1) / tile), p.splits);
    if (p.small) GATED_T(dt, hipLaunchKernelGGL((k_gated_tn<T, 1, 1>), grid, dim3(TPB), 0, s, (const T *)D, (const T *)x, rows, M, C, p.per_split, dw, db, part));
    else GATED_T(dt, hipLaunchKernelGGL((k_gated_tn<T, 2, 2>), grid, dim3(TPB), 0, s, (const T *)D, (const T *)x, rows, M, C, p.per_split, dw, db, part));
    if (part) {
        const size_t n = (size_t)M * C, all = n + (db ? M : 0);
        if (n % 4 == 0 && M % 4 == 0) hipLaunchKernelGGL(k_gated_tn_join<4>, dim3((unsigned)((all / 4 + TPB - 1) / TPB)), dim3(TPB), 0, s, part, p.splits, n, dw, (size_t)M, db);
        else hipLaunchKernelGGL(k_gated_tn_join<1>, dim3((unsigned)((all + TPB - 1) / TPB)), dim3(TPB), 0, s, part, p.splits, n, dw, (size_t)M, db);
    }
    return hipGetLastError();
}

}  // namespace bapipe
