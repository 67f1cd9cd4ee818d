// Attention, backward, the gradients of keys and values: a block owns keys and streams the queries that see them, of every query head
// that shares the key head.  No atomics: sums have one order.
//   dv = p^T dout, dk = ds^T q / sqrt(d)
#include "attention_common.h"

namespace bapipe {
namespace {

// Float heads of more than 128 channels would need more registers than there are: their blocks own half of the gradients' columns, two to a key
template <class T, int DP> constexpr int kDkvHalves = DP * (int)sizeof(T) > 768 ? 2 : 1;

template <class T, int DP, bool VEC, bool EXTRA, bool HALF>
__global__ __launch_bounds__(AT_TPB, (DP * (int)sizeof(T) <= 256 ? 2 : 1)) void k_attention_dkv(AttnArgs p)
{
    constexpr int R = HALF && DP >= 128 ? 32 : 0;        // three operands
    typedef AtTile<T, DP, R> Tile;
    typedef std::conditional_t<HALF, half_t, T> S;
    typedef AtTile<S, DP, R> STile;
    constexpr int HALVES = kDkvHalves<T, DP>, ND = DP / 32 / HALVES, SUBS = Tile::ROWS / 32, STREAMS = HALF ? 3 : 2;
    static_assert(Tile::ROWS <= kAttnTile && kAttnTile % Tile::ROWS == 0, "");
    extern __shared__ __align__(256) unsigned char smem[];
    // of the rows of a tile, twice: lse, dout . o, span, scale
    __shared__ __align__(16) float row_scale[2][HALF ? Tile::ROWS : 4];
    __shared__ __align__(16) float row_lse[2][Tile::ROWS], row_dsum[2][Tile::ROWS];
    __shared__ __align__(16) int row_first[2][Tile::ROWS], row_end[2][Tile::ROWS];
    __shared__ int2 block_range[AT_WAVES];
    const AttnShape &s = p.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
    const int d = s.d, stride = s.stride(), per = s.heads / s.groups, ostride = s.heads * d;
    const AtBlock b = at_block(s);
    // with a causal mask the first keys have the most queries
    const int half = b.rest % HALVES, split = b.rest / HALVES % p.splits, key0 = b.rest / HALVES / p.splits * AT_ROWS;
    const int wave0 = key0 + 32 * wave, k = wave0 + (lane & 31);
    const int sstride = HALF ? (s.heads + s.groups) * d : stride;
    const T *base = (const T *)p.qk + (size_t)b.n * s.T * stride;
    const S *score_base = (const S *)(HALF ? p.half : p.qk) + (size_t)b.n * s.T * sstride;
    chunk16 key[Tile::STEPS], value[Tile::STEPS];
    at_own<S, DP, VEC>(key, k < s.T ? score_base + (size_t)k * sstride + (size_t)(s.heads + b.g) * d : nullptr, d, lane);
    at_own<T, DP, VEC>(value, k < s.T ? (const T *)p.v + ((size_t)b.n * s.T + k) * stride + (size_t)(s.heads + s.groups + b.g) * d : nullptr, d, lane);

    // tiles of queries, from the first that sees one of the block's keys to the last
    const int all_tiles = (s.T + Tile::ROWS - 1) / Tile::ROWS;
    int first = 0, end = all_tiles;
    const int4 *bounds = p.bounds + (size_t)b.n * ((s.T + kAttnTile - 1) / kAttnTile);
    if (s.mask == ATTN_CAUSAL) first = key0 / Tile::ROWS;
    if (s.mask == ATTN_SPANS) {
        first = all_tiles;
        end = 0;
        for (int i = tid; i < all_tiles; i += AT_TPB) {
            const int4 v = bounds[i * Tile::ROWS / kAttnTile];
            if (v.x < key0 + AT_ROWS && v.y > key0) {
                first = min(first, i);
                end = i + 1;
            }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            first = min(first, __shfl_xor(first, o, 64));
            end = max(end, __shfl_xor(end, o, 64));
        }
        if (lane == 0) block_range[wave] = {first, end};
        __syncthreads();
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) {
            first = min(first, block_range[w].x);
            end = max(end, block_range[w].y);
        }
    }
    first = __builtin_amdgcn_readfirstlane(first);
    end = __builtin_amdgcn_readfirstlane(end);
    const int of_head = end > first ? end - first : 0, total = of_head * per;
    const int begin = (int)((long long)total * split / p.splits), stop = (int)((long long)total * (split + 1) / p.splits);

    const lds_addr_of lds(smem);
    const AtStream<T, DP, VEC, R> queries(stride, tid), gradients(ostride, tid);
    const AtStream<S, DP, VEC, R> score_queries(sstride, tid);
    const float own_scale = HALF && k < s.T ? p.half_scale[((size_t)(s.heads + b.g) * s.N + b.n) * s.T + k] : 1.0f;
    float next_lse = 0.0f, next_dsum = 0.0f, next_scale = 0.0f;
    int2 next_span = {0, 0};
    // head and tile of the loads that are under way; counted up, so that addresses stay scalar
    int next_head = 0, next_tile = 0;
    if (begin < stop) {
        next_head = __builtin_amdgcn_readfirstlane(b.g * per + begin / of_head);
        next_tile = __builtin_amdgcn_readfirstlane(first + begin % of_head);
    }
    auto fill = [&](int it) {
        const int head = next_head, q0 = next_tile * Tile::ROWS;
        if (tid < Tile::ROWS) {
            const int q = q0 + tid;
            next_span = at_span(p, b.n, q);
            const size_t at = ((size_t)b.n * s.heads + head) * s.T + q;
            next_lse = q < s.T ? p.lse[at] : __builtin_inff();
            next_dsum = q < s.T ? p.dsum[at] : 0.0f;
            if (HALF) next_scale = q < s.T ? p.half_scale[((size_t)head * s.N + b.n) * s.T + q] : 0.0f;
        }
        unsigned char *to = smem + (it & 1) * STREAMS * Tile::BYTES;
        queries.fill(to, lds, base + (size_t)q0 * stride + (size_t)head * d, s.T - q0, stride, d, tid);
        gradients.fill(to + Tile::BYTES, lds, (const T *)p.dout + ((size_t)b.n * s.T + q0) * ostride + (size_t)head * d, s.T - q0, ostride, d, tid);
        if (HALF) score_queries.fill(to + 2 * Tile::BYTES, lds, score_base + (size_t)q0 * sstride + (size_t)head * d, s.T - q0, sstride, d, tid);
    };
    f32x16_t dk[ND] = {}, dv[ND] = {};
    AtScore score = {};
    int head_of = -1;
    if (begin < stop) fill(begin);
    for (int it = begin; it < stop; ++it) {
        const int at = it & 1;
        if (tid < Tile::ROWS) {
            row_lse[at][tid] = next_lse;
            row_dsum[at][tid] = next_dsum;
            if (HALF) row_scale[at][tid] = next_scale;
            row_first[at][tid] = next_span.x;
            row_end[at][tid] = next_span.y;
        }
        WAIT_VMCNT(0);
        at_barrier();
        const int head = next_head, q0 = next_tile * Tile::ROWS;
        if (head != head_of) score = at_score(s, head_of = head);
        if (++next_tile == end) {
            next_tile = first;
            ++next_head;
        }
        if (it + 1 < stop) fill(it + 1);
        // what the tile's queries see, and whether all of them see all of the wave's keys
        bool none = wave0 >= s.T, whole = q0 + Tile::ROWS <= s.T;
        if (s.mask == ATTN_CAUSAL) {
            none |= q0 + Tile::ROWS <= wave0;
            whole &= q0 >= wave0 + 31;
        } else if (s.mask == ATTN_SPANS) {
            const int4 v = bounds[q0 / kAttnTile];
            none |= v.x >= wave0 + 32 || v.y <= wave0;
            whole &= v.z <= wave0 && v.w >= wave0 + 32;
        }
        if (none) continue;
        const unsigned char *query = smem + at * STREAMS * Tile::BYTES, *dout = query + Tile::BYTES, *score_query = HALF ? dout + Tile::BYTES : query;
#pragma unroll 1
        for (int u = 0; u < SUBS; ++u) {
            const f32x16_t w = at_rows<S, STile>(score_query, 32 * u, key, lane), dw = at_rows<T, Tile>(dout, 32 * u, value, lane);
            float x[16], ds[16], slope[16];
            const int r = 32 * u + 4 * h;                                // rows of a register's four: r + 8 g
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 dsum = *(const float4 *)&row_dsum[at][r + 8 * g];
                float4 scale = {1.0f, 1.0f, 1.0f, 1.0f};
                if (HALF) scale = *(const float4 *)&row_scale[at][r + 8 * g];
                const float less[4] = {dsum.x, dsum.y, dsum.z, dsum.w}, by_row[4] = {scale.x, scale.y, scale.z, scale.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[4 * g + j] = HALF ? w[4 * g + j] * by_row[j] : w[4 * g + j];
                    ds[4 * g + j] = dw[4 * g + j] - less[j];
                }
            }
            const float by = score.scale * own_scale;
            if (EXTRA) at_bend<T, true>(x, score, by, (float)(k - (q0 + r)), slope);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 lse = *(const float4 *)&row_lse[at][r + 8 * g];
                const float less[4] = {lse.x, lse.y, lse.z, lse.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * g + j] = __builtin_amdgcn_exp2f(fmaf(x[4 * g + j], EXTRA ? 1.0f : by, -less[j]));
            }
            if (!whole)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int4 from = *(const int4 *)&row_first[at][r + 8 * g], to = *(const int4 *)&row_end[at][r + 8 * g];
                    const int f[4] = {from.x, from.y, from.z, from.w}, e[4] = {to.x, to.y, to.z, to.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[4 * g + j] = k >= f[j] && k < e[j] ? x[4 * g + j] : 0.0f;
                }
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] = EXTRA ? x[i] * ds[i] * slope[i] : x[i] * ds[i];
            at_columns<T, Tile, ND>(dv, dout, 32 * u, half * ND, AtWeights<T>(x), lane);
            at_columns<T, Tile, ND>(dk, query, 32 * u, half * ND, AtWeights<T>(ds), lane);
        }
    }
    if (k >= s.T) return;
    if (p.splits > 1) {
        float *to = p.part + ((((size_t)split * s.N + b.n) * s.groups + b.g) * s.T + k) * 2 * d;
        at_store<float, VEC, ND>(to, d, half * ND, dk, s.scale, lane);
        at_store<float, VEC, ND>(to + d, d, half * ND, dv, 1.0f, lane);
        return;
    }
    const size_t row = (size_t)b.n * s.T + k, at_k = row * stride + (size_t)(s.heads + b.g) * d;
    if (p.dqk_float) at_store<float, VEC, ND>(p.dqk_float + row * (s.heads + s.groups) * d + (size_t)(s.heads + b.g) * d, d, half * ND, dk, s.scale, lane);
    else at_store<T, VEC, ND>((T *)p.dqk + at_k, d, half * ND, dk, s.scale, lane);
    at_store<T, VEC, ND>((T *)p.dv + at_k + (size_t)s.groups * d, d, half * ND, dv, 1.0f, lane);
}

// The sums of all splits, an element a thread
template <class T> __global__ __launch_bounds__(256) void k_attention_join(AttnArgs p)
{
    const AttnShape &s = p.s;
    const size_t n = (size_t)s.N * s.groups * s.T * 2 * s.d, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float sum = 0.0f;
    for (int k = 0; k < p.splits; ++k) sum += p.part[k * n + i];
    const int e = (int)(i % s.d), which = (int)(i / s.d % 2);
    const size_t row = i / (2 * s.d);                              // [N][groups][T]
    const int t = (int)(row % s.T), g = (int)(row / s.T % s.groups);
    const size_t at = (row / s.T / s.groups * s.T + t) * s.stride() + (size_t)(s.heads + g) * s.d + e;
    if (which) ((T *)p.dv)[at + (size_t)s.groups * s.d] = from_f32<T>(sum);
    else if (p.dqk_float) p.dqk_float[((row / s.T / s.groups * s.T + t) * (s.heads + s.groups) + s.heads + g) * s.d + e] = sum;
    else ((T *)p.dqk)[at] = from_f32<T>(sum);
}

template <class T, int DP, bool VEC, bool EXTRA, bool HALF> struct Keys {
    static hipError_t go(const AttnArgs &a, hipStream_t stream)
    {
        constexpr int smem = HALF ? 6 * AtTile<T, DP, DP >= 128 ? 32 : 0>::BYTES : 4 * AtTile<T, DP>::BYTES;
        return at_launch(k_attention_dkv<T, DP, VEC, EXTRA, HALF>, a.s.N * a.s.groups * ((a.s.T + AT_ROWS - 1) / AT_ROWS) * a.splits * kDkvHalves<T, DP>, smem, a,
                         stream);
    }
};

// In how many parts the queries of the keys' sums are taken: few keys leave units idle
int key_splits(const AttnShape &s, int compute_units)
{
    (void)compute_units;
    return 1;
}

}  // namespace

hipError_t attention_dkv(int dt, const AttnArgs &a, hipStream_t s)
{
    const hipError_t e = at_dispatch<Keys>(dt, a, s);
    if (e != hipSuccess || a.splits == 1) return e;
    const size_t n = (size_t)a.s.N * a.s.groups * a.s.T * 2 * a.s.d;
    const dim3 grid((unsigned)((n + 255) / 256));
    if (dt == DT_F32) hipLaunchKernelGGL((k_attention_join<float>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attention_join<bf16_t>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t attention_workspace(int dt, const AttnShape &a, int compute_units)
{
    (void)dt;
    const int splits = key_splits(a, compute_units);
    const size_t rows = ((size_t)a.N * a.heads * a.T * sizeof(float) + 255) / 256 * 256;
    return rows + (splits > 1 ? (size_t)splits * a.N * a.groups * a.T * 2 * a.d * sizeof(float) : 0);
}

hipError_t attention_bwd(int dt, AttnArgs a, void *workspace, int compute_units, hipStream_t s)
{
    a.dsum = (float *)workspace;
    a.part = (float *)((char *)workspace + ((size_t)a.s.N * a.s.heads * a.s.T * sizeof(float) + 255) / 256 * 256);
    a.splits = key_splits(a.s, compute_units);
    const hipError_t e = attention_dq(dt, a, s);
    return e == hipSuccess ? attention_dkv(dt, a, s) : e;
}

}  // namespace bapipe
