// Layer norm over the channels of every position of an NHWC tensor, read as a matrix [rows][C].
//   mean = sum x / C, var = sum (x - mean)^2 / C, inv = 1 / sqrt(var + eps), xhat = (x - mean) inv, y = gamma xhat + beta
//   a = gamma dy;  dx = inv (a - sum a / C - xhat sum(a xhat) / C);  dgamma += sum over rows of dy xhat;  dbeta += sum over rows of dy
// Everything between a load and a store is float; mean and inv of every row are kept for the backward pass.
#include "dev_common.h"
#include "kernels.h"

namespace bapipe {
namespace {

constexpr int TPB = 256;

// sum over the block, for all its threads
__device__ __forceinline__ float block_sum(float v, float *lds)
{
    v = wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < TPB / 64; ++w) sum += lds[w];
    return sum;
}

// a block takes rows blockIdx.x, blockIdx.x + gridDim.x, ...
template <class T>
__global__ __launch_bounds__(TPB) void k_layernorm_fwd(const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                       float eps, T *__restrict__ y, float *__restrict__ stats, int rows, int C)
{
    __shared__ float lds[TPB / 64];
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
    const T *xr = x + (size_t)row * C;
    float sum = 0.0f;
    for (int c = threadIdx.x; c < C; c += TPB) sum += to_f32(xr[c]);
    const float mean = block_sum(sum, lds) / C;
    float sq = 0.0f;
    for (int c = threadIdx.x; c < C; c += TPB) {
        const float d = to_f32(xr[c]) - mean;
        sq += d * d;
    }
    const float inv = 1.0f / sqrtf(block_sum(sq, lds) / C + eps);
    for (int c = threadIdx.x; c < C; c += TPB)
        y[(size_t)row * C + c] = from_f32<T>((to_f32(xr[c]) - mean) * inv * gamma[c] + beta[c]);
    if (threadIdx.x == 0) {
        stats[row] = mean;
        stats[rows + row] = inv;
    }
    }
}

template <class T>
__global__ __launch_bounds__(TPB) void k_layernorm_dx(const T *x, const T *dy, const float *__restrict__ gamma, const float *__restrict__ stats,
                                                      T *dx, const T *old, const T *gate, int rows, int C)
{
    __shared__ float lds[TPB / 64];
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
    const size_t at = (size_t)row * C;
    const float mean = stats[row], inv = stats[rows + row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < C; c += TPB) {
        const float a = to_f32(dy[at + c]) * gamma[c];
        s1 += a;
        s2 += a * ((to_f32(x[at + c]) - mean) * inv);
    }
    s1 = block_sum(s1, lds) / C;
    s2 = block_sum(s2, lds) / C;
    for (int c = threadIdx.x; c < C; c += TPB) {
        const float a = to_f32(dy[at + c]) * gamma[c], xhat = (to_f32(x[at + c]) - mean) * inv;
        dx[at + c] = grad_out<T>(inv * (a - s1 - xhat * s2), old != nullptr, old ? old[at + c] : from_f32<T>(0.0f), gate != nullptr,
                                 gate ? gate[at + c] : from_f32<T>(0.0f));
    }
    }
}

// part[chunk][0 | 1][C]: sums of dy xhat and of dy over the chunk's rows, a column per thread
template <class T>
__global__ __launch_bounds__(TPB) void k_layernorm_columns(const T *__restrict__ x, const T *__restrict__ dy, const float *__restrict__ stats,
                                                           float *__restrict__ part, int rows, int C, int rows_per_chunk)
{
    const int c = blockIdx.x * TPB + threadIdx.x;
    if (c >= C) return;
    const int r0 = blockIdx.y * rows_per_chunk, r1 = r0 + rows_per_chunk < rows ? r0 + rows_per_chunk : rows;
    float g = 0.0f, b = 0.0f;
    for (int r = r0; r < r1; ++r) {
        const float d = to_f32(dy[(size_t)r * C + c]);
        g += d * ((to_f32(x[(size_t)r * C + c]) - stats[r]) * stats[rows + r]);
        b += d;
    }
    part[(size_t)blockIdx.y * 2 * C + c] = g;
    part[((size_t)blockIdx.y * 2 + 1) * C + c] = b;
}

// dgamma += , dbeta += the sums of all chunks, in chunk order
__global__ __launch_bounds__(TPB) void k_layernorm_params(const float *__restrict__ part, int chunks, int C, float *dgamma, float *dbeta)
{
    const int i = blockIdx.x * TPB + threadIdx.x;
    if (i >= 2 * C) return;
    double sum = 0.0;
    for (int k = 0; k < chunks; ++k) sum += part[(size_t)k * 2 * C + i];
    float *out = i < C ? dgamma + i : dbeta + (i - C);
    *out += (float)sum;
}

unsigned grid_of(int rows) { return rows < 1 << 20 ? rows : 1 << 20; }
int rows_per_chunk(int rows) { return rows < 64 * 256 ? 64 : (rows + 255) / 256; }
int chunks_of(int rows) { return (rows + rows_per_chunk(rows) - 1) / rows_per_chunk(rows); }

}  // namespace

size_t layernorm_workspace(int rows, int C) { return (size_t)chunks_of(rows) * 2 * C * sizeof(float); }

hipError_t layernorm_fwd(int dt, const void *x, const float *gamma, const float *beta, float eps, void *y, float *stats, int rows, int C, hipStream_t s)
{
    if (dt == DT_F32)
        hipLaunchKernelGGL((k_layernorm_fwd<float>), dim3(grid_of(rows)), dim3(TPB), 0, s, (const float *)x, gamma, beta, eps, (float *)y, stats, rows, C);
    else
        hipLaunchKernelGGL((k_layernorm_fwd<bf16_t>), dim3(grid_of(rows)), dim3(TPB), 0, s, (const bf16_t *)x, gamma, beta, eps, (bf16_t *)y, stats, rows, C);
    return hipGetLastError();
}

template <class T>
static hipError_t layernorm_bwd_t(const T *x, const T *dy, const float *gamma, const float *stats, T *dx, float *dgamma, float *dbeta, GradEpi epi,
                                  int rows, int C, float *part, hipStream_t s)
{
    // before dx, which may take the place of dy
    const int per = rows_per_chunk(rows), chunks = chunks_of(rows);
    hipLaunchKernelGGL((k_layernorm_columns<T>), dim3((C + TPB - 1) / TPB, chunks), dim3(TPB), 0, s, x, dy, stats, part, rows, C, per);
    hipLaunchKernelGGL(k_layernorm_params, dim3((2 * C + TPB - 1) / TPB), dim3(TPB), 0, s, part, chunks, C, dgamma, dbeta);
    const T *old = epi.accum ? (const T *)(epi.accum_from ? epi.accum_from : dx) : nullptr;
    if (dx)
        hipLaunchKernelGGL((k_layernorm_dx<T>), dim3(grid_of(rows)), dim3(TPB), 0, s, x, dy, gamma, stats, dx, old, (const T *)epi.gate, rows, C);
    return hipGetLastError();
}

hipError_t layernorm_bwd(int dt, const void *x, const void *dy, const float *gamma, const float *stats, void *dx, float *dgamma, float *dbeta,
                         GradEpi epi, int rows, int C, void *workspace, hipStream_t s)
{
    if (dt == DT_F32)
        return layernorm_bwd_t((const float *)x, (const float *)dy, gamma, stats, (float *)dx, dgamma, dbeta, epi, rows, C, (float *)workspace, s);
    return layernorm_bwd_t((const bf16_t *)x, (const bf16_t *)dy, gamma, stats, (bf16_t *)dx, dgamma, dbeta, epi, rows, C, (float *)workspace, s);
}

}  // namespace bapipe
