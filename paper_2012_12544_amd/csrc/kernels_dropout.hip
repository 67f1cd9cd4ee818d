// Dropout whose mask is computed where it is needed, forward and backward, and stored nowhere.
#include "dev_common.h"
#include "kernels.h"

namespace bapipe {
namespace {

constexpr int TPB = 256;

// Four random words of a 128-bit counter under a 64-bit key: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel
// random numbers: as easy as 1, 2, 3", SC'11).
struct words4 {
    uint32_t w[4];
};
__device__ __forceinline__ words4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// y[e] = word(e) >= threshold ? x[e] * scale : 0, sixteen bytes a thread: four elements of one counter, or eight of two.
// state: seed (low, high word), number of the mini-batch - read from memory, so that a captured launch draws anew when it is replayed
// HBM bounds it: twenty products of 32 x 32 bits for four words are what the vector unit has time for beside 4 bytes an element
// (seven rounds instead of ten took as long).  What is read and written once passes by the caches: 2^27 bf16 elements, us: 125 with ordinary
// accesses, 99 with such stores, 85 (6.3 TB/s) with such loads too.  Loads of up to 8 MB, which the kernel before has left in the
// caches, stay ordinary ones (3.3 M elements: 5.7, and 5.9 with the others).
enum { PLAIN, GRADIENT, SUM };       // SUM: a residual sum y = [relu](round(dropped x) + old)
constexpr size_t kCached = 8u << 20;
typedef uint32_t any16 __attribute__((ext_vector_type(4), aligned(2)));          // 16 bytes at any address of an element
template <class T> struct DropArgs {
    const T *x;
    T *y;
    const T *old, *gate;      // GRADIENT: see grad_out(); SUM: old is the other summand
    size_t n;
    uint32_t threshold;
    float scale;
    const uint32_t *state;
    uint32_t layer, mb;
    int relu;
};

template <class T, int MODE, bool CACHED>
__global__ __launch_bounds__(TPB) void k_dropout(DropArgs<T> p)
{
    constexpr int V = 16 / sizeof(T);
    struct vec {
        T e[V];
    };
    const size_t i = (size_t)blockIdx.x * TPB + threadIdx.x, e0 = i * V;
    if (e0 >= p.n) return;
    // at any address of T; the tensor's last elements one by one
    const int left = p.n - e0 < V ? (int)(p.n - e0) : V;
    auto load = [&](const T *from) {
        vec v;
        if (left == V) v = __builtin_bit_cast(vec, CACHED ? *(const any16 *)(from + e0) : __builtin_nontemporal_load((const any16 *)(from + e0)));
        else
#pragma unroll
            for (int j = 0; j < V; ++j) v.e[j] = j < left ? from[e0 + j] : T{};
        return v;
    };
    const vec x = load(p.x);
    vec old = {}, gate = {}, y;
    if (MODE == SUM || (MODE == GRADIENT && p.old)) old = load(p.old);
    if (MODE == GRADIENT && p.gate) gate = load(p.gate);
    const uint32_t k0 = p.state[0], k1 = p.state[1], mini_batch = p.state[2];
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
        const words4 r = philox((uint32_t)(i * (V / 4) + q), p.layer, p.mb, mini_batch, k0, k1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = q * 4 + j;
            const float v = r.w[j] >= p.threshold ? to_f32(x.e[e]) * p.scale : 0.0f;
            if (MODE == PLAIN) y.e[e] = from_f32<T>(v);
            else if (MODE == GRADIENT) y.e[e] = grad_out<T>(v, p.old != nullptr, old.e[e], p.gate != nullptr, gate.e[e]);
            else {
                const float sum = round_to<T>(v) + to_f32(old.e[e]);
                y.e[e] = from_f32<T>(p.relu ? fmaxf(sum, 0.0f) : sum);
            }
        }
    }
    if (left == V) __builtin_nontemporal_store(__builtin_bit_cast(any16, y), (any16 *)(p.y + e0));
    else
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < left) p.y[e0 + j] = y.e[j];
}

__global__ void k_dropout_set(uint32_t *state, uint32_t low, uint32_t high, uint32_t mini_batch)
{
    state[0] = low;
    state[1] = high;
    state[2] = mini_batch;
}
__global__ void k_dropout_next(uint32_t *state) { state[2] += 1; }

}  // namespace

template <class T, int MODE>
static hipError_t launch(const void *x, void *y, const void *old, const void *gate, int relu, size_t n, float p, const uint32_t *state, uint32_t layer,
                         uint32_t mb, hipStream_t s)
{
    if (n == 0) return hipSuccess;
    // dropped where a word is below 2^32 p, which a probability just under one would round up to
    const double t = (double)p * 4294967296.0 + 0.5;
    DropArgs<T> a{(const T *)x, (T *)y, (const T *)old, (const T *)gate, n, t < 4294967295.0 ? (uint32_t)t : 0xFFFFFFFFu,
                  (float)(1.0 / (1.0 - (double)p)), state, layer, mb, relu};
    constexpr size_t per_block = TPB * (16 / sizeof(T));
    const dim3 grid((unsigned)((n + per_block - 1) / per_block));
    if (n * sizeof(T) <= kCached) hipLaunchKernelGGL((k_dropout<T, MODE, true>), grid, dim3(TPB), 0, s, a);
    else hipLaunchKernelGGL((k_dropout<T, MODE, false>), grid, dim3(TPB), 0, s, a);
    return hipGetLastError();
}

hipError_t dropout(int dt, const void *x, void *y, GradEpi epi, size_t n, float p, const uint32_t *state, uint32_t layer, uint32_t mb,
                   hipStream_t s)
{
    const void *old = epi.accum ? (epi.accum_from ? epi.accum_from : y) : nullptr;
    const bool plain = !old && !epi.gate;
    if (dt == DT_F32)
        return plain ? launch<float, PLAIN>(x, y, nullptr, nullptr, 0, n, p, state, layer, mb, s)
                     : launch<float, GRADIENT>(x, y, old, epi.gate, 0, n, p, state, layer, mb, s);
    return plain ? launch<bf16_t, PLAIN>(x, y, nullptr, nullptr, 0, n, p, state, layer, mb, s)
                 : launch<bf16_t, GRADIENT>(x, y, old, epi.gate, 0, n, p, state, layer, mb, s);
}

hipError_t dropout_add(int dt, const void *x, const void *other, void *y, int relu, size_t n, float p, const uint32_t *state, uint32_t layer,
                       uint32_t mb, hipStream_t s)
{
    if (dt == DT_F32) return launch<float, SUM>(x, y, other, nullptr, relu, n, p, state, layer, mb, s);
    return launch<bf16_t, SUM>(x, y, other, nullptr, relu, n, p, state, layer, mb, s);
}

hipError_t dropout_set(uint32_t *state, uint64_t seed, uint32_t mini_batch, hipStream_t s)
{
    hipLaunchKernelGGL(k_dropout_set, dim3(1), dim3(1), 0, s, state, (uint32_t)seed, (uint32_t)(seed >> 32), mini_batch);
    return hipGetLastError();
}

hipError_t dropout_next(uint32_t *state, hipStream_t s)
{
    hipLaunchKernelGGL(k_dropout_next, dim3(1), dim3(1), 0, s, state);
    return hipGetLastError();
}

}  // namespace bapipe
