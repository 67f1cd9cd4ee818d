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

// y[e] = word(e) >= threshold ? x[e] * scale : 0, for four elements of one counter a thread.
// state: seed (low, high word), number of the mini-batch - read from memory, so that a captured launch draws anew when it is replayed
template <class T>
__global__ __launch_bounds__(TPB) void k_dropout(const T *x, T *y, const T *old, const T *gate, size_t n, uint32_t threshold, float scale,
                                                 const uint32_t *__restrict__ state, uint32_t layer, uint32_t mb)
{
    const size_t i = (size_t)blockIdx.x * TPB + threadIdx.x, e0 = i * 4;
    if (e0 >= n) return;
    const words4 r = philox((uint32_t)i, layer, mb, state[2], state[0], state[1]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const size_t e = e0 + j;
        if (e >= n) break;
        const float v = r.w[j] >= threshold ? to_f32(x[e]) * scale : 0.0f;
        y[e] = grad_out<T>(v, old != nullptr, old ? old[e] : from_f32<T>(0.0f), gate != nullptr, gate ? gate[e] : from_f32<T>(0.0f));
    }
}

__global__ void k_dropout_set(uint32_t *state, uint32_t low, uint32_t high, uint32_t mini_batch)
{
    state[0] = low;
    state[1] = high;
    state[2] = mini_batch;
}
__global__ void k_dropout_next(uint32_t *state) { state[2] += 1; }

}  // namespace

hipError_t dropout(int dt, const void *x, void *y, GradEpi epi, size_t n, float p, const uint32_t *state, uint32_t layer, uint32_t mb,
                   hipStream_t s)
{
    if (n == 0) return hipSuccess;
    // dropped where a word is below 2^32 p, which a probability just under one would round up to
    const double t = (double)p * 4294967296.0 + 0.5;
    const uint32_t threshold = t < 4294967295.0 ? (uint32_t)t : 0xFFFFFFFFu;
    const float scale = (float)(1.0 / (1.0 - (double)p));
    const void *old = epi.accum ? (epi.accum_from ? epi.accum_from : y) : nullptr;
    const dim3 grid((unsigned)((n + 4 * TPB - 1) / (4 * TPB)));
    if (dt == DT_F32)
        hipLaunchKernelGGL((k_dropout<float>), grid, dim3(TPB), 0, s, (const float *)x, (float *)y, (const float *)old, (const float *)epi.gate, n,
                           threshold, scale, state, layer, mb);
    else
        hipLaunchKernelGGL((k_dropout<bf16_t>), grid, dim3(TPB), 0, s, (const bf16_t *)x, (bf16_t *)y, (const bf16_t *)old, (const bf16_t *)epi.gate,
                           n, threshold, scale, state, layer, mb);
    return hipGetLastError();
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
