// Attention, backward, the queries' gradients: scores and probabilities again from the stored logarithm of each query's sum.
//   p = 2^(score - lse), ds = p (dout v^T - dout . o), dq = ds k / sqrt(d)
// 4 x 4096 positions, causal, 32 / 8 heads of 128, bf16: 872 us, 946 TFLOP/s of its three products, 57 % of the cycles.  One of them
// is the forward pass's again: to keep it would be to write and read 2 bytes for each of 1.1e9 pairs.
#include "attention_common.h"

namespace bapipe {
namespace {

template <class T, int DP, bool VEC, bool EXTRA, bool HALF, int KS>
__global__ __launch_bounds__(AT_TPB, (DP * (int)sizeof(T) <= 256 ? 2 : 1)) void k_attention_dq(AttnArgs p)
{
    typedef AtTile<T, DP> Tile;
    typedef std::conditional_t<HALF, half_t, T> S;       // queries and keys
    typedef AtTile<S, DP> STile;
    constexpr int ND = DP / 32, SUBS = Tile::ROWS / 32;
    extern __shared__ __align__(256) unsigned char smem[];
    __shared__ int2 block_range[AT_WAVES];
    const AttnShape &s = p.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, ks = wave % KS;
    const int d = s.d, stride = s.stride(), per = s.heads / s.groups;
    const AtBlock b = at_block(s);
    const int head = b.g * per + b.rest % per, q0 = at_query_block<KS>(p, b.n, b.rest / per) * (AT_ROWS / KS);
    const int q = q0 + 32 * (wave / KS) + (lane & 31);
    const int sstride = HALF ? (s.heads + s.groups) * d : stride;
    const S *base = (const S *)(HALF ? p.half : p.qk) + (size_t)b.n * s.T * sstride, *keys = base + (size_t)(s.heads + b.g) * d;
    const T *values = (const T *)p.v + (size_t)b.n * s.T * stride + (size_t)(s.heads + s.groups + b.g) * d;
    const float *key_scale = HALF ? p.half_scale + ((size_t)(s.heads + b.g) * s.N + b.n) * s.T : nullptr;
    const size_t at_o = ((size_t)b.n * s.T + q) * s.heads * d + (size_t)head * d, at_row = ((size_t)b.n * s.heads + head) * s.T + q;

    const int2 span = at_span(p, b.n, q);
    const bool sees = span.x < span.y;
    chunk16 query[Tile::STEPS], dout[Tile::STEPS];
    at_own<S, DP, VEC>(query, sees ? base + (size_t)q * sstride + (size_t)head * d : nullptr, d, lane);
    at_own<T, DP, VEC>(dout, sees ? (const T *)p.dout + at_o : nullptr, d, lane);
    float dsum = 0.0f;
    {
        chunk16 o[Tile::STEPS];
        at_own<T, DP, VEC>(o, sees ? (const T *)p.o + at_o : nullptr, d, lane);
        uint2 low[Tile::STEPS];
        if (sizeof(T) == 2)
#pragma unroll
            for (int c = 0; c < Tile::STEPS; ++c) {
                const int e0 = (2 * c + h) * 8;
                low[c] = {0, 0};
                if constexpr (VEC) {
                    if (sees && e0 < d) low[c] = *(const uint2 *)(p.o_low + at_o + e0);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t b = sees && e0 + j < d ? (uint8_t)p.o_low[at_o + e0 + j] : 0;
                        (j < 4 ? low[c].x : low[c].y) |= b << 8 * (j & 3);
                    }
                }
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < Tile::STEPS; ++c)
#pragma unroll
            for (int j = 0; j < Tile::EPC; ++j) {
                float of = chunk_value<T>(o[c], j);
                if (sizeof(T) == 2) of = at_whole(__float_as_uint(of) >> 16, (int)(int8_t)((j < 4 ? low[c].x : low[c].y) >> 8 * (j & 3)));
                dsum = fmaf(chunk_value<T>(dout[c], j), of, dsum);
            }
        dsum = at_halves_sum(dsum);
    }
    const float lse = sees ? p.lse[at_row] : __builtin_inff();
    if (ks == 0 && q < s.T && h == 0) p.dsum[at_row] = dsum;

    const AtRange range = at_wave_range(span);
    if (lane == 0) block_range[wave] = range.any;
    __syncthreads();
    int first = s.T, end = 0;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
        first = min(first, block_range[w].x);
        end = max(end, block_range[w].y);
    }
    first = __builtin_amdgcn_readfirstlane(first);
    end = __builtin_amdgcn_readfirstlane(end);

    const AtScore score = at_score(s, head);
    float by = score.scale;
    if (HALF && sees) by *= p.half_scale[((size_t)head * s.N + b.n) * s.T + q];
    const unsigned lds = at_lds(smem);
    AtStream<S, DP, VEC> key_stream(sstride, tid);
    AtStream<T, DP, VEC> value_stream(stride, tid);
    constexpr int SCALE_AT = 4 * Tile::BYTES;                // 64 words, twice
    auto fill = [&](int it) {
        const int k0 = first + it * Tile::ROWS;
        const int to = (it & 1) * 2 * Tile::BYTES;
        if (HALF && wave == 0) at_dma4(key_scale + k0, end - k0, lds + SCALE_AT + (it & 1) * 256, tid);
        key_stream.fill(smem, lds, to, keys + (size_t)k0 * sstride, end - k0, sstride, d, tid);
        value_stream.fill(smem, lds, to + Tile::BYTES, values + (size_t)k0 * stride, end - k0, stride, d, tid);
    };
    f32x16_t dq[ND] = {};
    float mult = HALF ? kAtRoom : 1.0f;
    const int tiles = (end - first + Tile::ROWS - 1) / Tile::ROWS;
    if (tiles > 0) fill(0);
    for (int it = 0; it < tiles; ++it) {
        WAIT_VMCNT(0);
        at_barrier();
        if (it + 1 < tiles) fill(it + 1);
        const int k0 = first + it * Tile::ROWS;
        if (k0 >= range.any.y || k0 + Tile::ROWS <= range.any.x) continue;
        const unsigned char *key = smem + (it & 1) * 2 * Tile::BYTES, *value = key + Tile::BYTES;
        const bool whole = k0 >= range.all.x && k0 + Tile::ROWS <= range.all.y;
#pragma unroll 1
        for (int u = ks; u < SUBS; u += KS) {
            f32x16_t w, dw;
            at_rows<S, STile>(w, key, 32 * u, query, d, lane);
            at_rows<T, Tile>(dw, value, 32 * u, dout, d, lane);
            float x[16], ds[16], slope[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = w[i];
                ds[i] = dw[i] - dsum;
            }
            if (HALF)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 r = *(const float4 *)(smem + SCALE_AT + (it & 1) * 256 + 4 * (32 * u + 8 * g + 4 * h));
                    x[4 * g] *= r.x; x[4 * g + 1] *= r.y; x[4 * g + 2] *= r.z; x[4 * g + 3] *= r.w;
                }
            if (EXTRA) at_bend<T, true>(x, score, by, (float)(q - (k0 + 32 * u + 4 * h)), slope);
            const float unit = EXTRA ? 1.0f : by;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], unit, -lse));
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = k0 + 32 * u + 8 * (i >> 2) + 4 * h + (i & 3);
                    x[i] = k >= span.x && k < span.y ? x[i] : 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] = EXTRA ? x[i] * ds[i] * slope[i] : x[i] * ds[i];
            if (HALF) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 r = *(const float4 *)(smem + SCALE_AT + (it & 1) * 256 + 4 * (32 * u + 8 * g + 4 * h));
                    ds[4 * g] *= r.x; ds[4 * g + 1] *= r.y; ds[4 * g + 2] *= r.z; ds[4 * g + 3] *= r.w;
                }
                at_fit(ds, mult, dq);
            }
            at_columns<S, STile>(dq, key, 32 * u, 0, AtWeights<S>(ds), d, lane);
        }
    }
    unsigned char *own = smem + wave * kAtOwn<DP>;
    float by_mult = s.scale / mult;
    if constexpr (KS == 2) {
        float *theirs = (float *)(smem + wave / 2 * (64 * 16 * ND * 4));
        own = (unsigned char *)theirs;
        at_barrier();                                      // the tiles are read
        if (ks) at_give(theirs, dq, by_mult, lane);
        at_barrier();
        if (ks) return;
        at_take(theirs, dq, by_mult, 1.0f, lane);
        by_mult = 1.0f;
    }
    if (VEC && sizeof(T) == 2 && !p.dqk_float) {
        if (KS == 1) at_barrier();                         // the tiles are read
        const int row0 = q0 + 32 * (wave / KS);
        if constexpr (VEC && sizeof(T) == 2)
            at_store_rows<DP, ND>(own, (T *)p.dqk + ((size_t)b.n * s.T + row0) * stride + (size_t)head * d, nullptr, stride, s.T - row0, d, dq,
                                  by_mult, lane);
        return;
    }
    if (q >= s.T) return;
    const size_t row = (size_t)b.n * s.T + q;
    if (p.dqk_float) at_store<float, VEC, ND>(p.dqk_float + row * (s.heads + s.groups) * d + (size_t)head * d, d, 0, dq, by_mult, lane);
    else at_store<T, VEC, ND>((T *)p.dqk + row * stride + (size_t)head * d, d, 0, dq, by_mult, lane);
}

template <class T, int DP, bool VEC, bool EXTRA, bool HALF> struct Queries {
    template <int KS> static hipError_t launch(const AttnArgs &a, hipStream_t stream)
    {
        constexpr int smem = std::max(4 * AtTile<T, DP>::BYTES + (HALF ? 512 : 0), sizeof(T) == 2 ? AT_WAVES * kAtOwn<DP> : 0);
        return at_launch(k_attention_dq<T, DP, VEC, EXTRA, HALF, KS>, a.s.N * a.s.heads * ((a.s.T + AT_ROWS / KS - 1) / (AT_ROWS / KS)), smem, a, stream);
    }
    static hipError_t go(const AttnArgs &a, hipStream_t stream)
    {
        if constexpr (kAtShares<T, DP>)
            if (at_shares(a, (long long)a.s.N * a.s.heads * ((a.s.T + AT_ROWS - 1) / AT_ROWS))) return launch<2>(a, stream);
        return launch<1>(a, stream);
    }
};

}  // namespace

hipError_t attention_dq(int dt, const AttnArgs &a, hipStream_t s) { return at_dispatch<Queries>(dt, a, s); }

}  // namespace bapipe
