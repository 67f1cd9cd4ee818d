// Attention, backward, the gradients of keys and values: a block owns keys and streams the queries that see them, of every query head
// that shares the key head.  No atomics: sums have one order.
//   dv = p^T dout, dk = ds^T q / sqrt(d)
// 4 x 4096 positions, causal, 32 / 8 heads of 128, bf16: 1173 us, 938 TFLOP/s of its four products, 59 % of the cycles.  Two waves a SIMD hold
// both sums, key and value of 32 rows in 256 registers each; 64 rows a wave, at one wave, halve the LDS reads and were slower (1842 us where this
// form took 1515).
#include "attention_common.h"

namespace bapipe {
namespace {

// Float heads of more than 128 channels, and 16-bit floats of 256, would need more registers than there are: their blocks own half of the gradients'
// columns, two to a key, and make the scores twice.  A mini-batch of 2 x 4 x 2048 positions of 16 / 8 heads of 256 behind a ROTARY, us:
// 4485 whole, with 245 registers spilled, 3022 so.
template <class T, int DP, bool HALF> constexpr int kDkvHalves = DP * (int)sizeof(T) > 768 || (HALF && DP > 192) ? 2 : 1;

// Rows of a tile, 0: what fits.  16-bit floats of 128 channels (4 x 2048 positions, causal, 16 / 2 heads), us: with 64 rows, 66 registers spilled,
// 286, with 32 and 36 of them 261; one wave a SIMD, which spills none, 281.  Now, with 32, 29 are spilled: 246.
template <int DP, bool EXTRA, bool HALF, int KS> constexpr int kDkvRows = KS == 1 && HALF && !EXTRA && DP == 128 ? 32 : 0;

// Blocks that the launch bounds let a unit hold, and those that fit: float heads of up to 64 channels take 251 registers
template <class T, int DP, bool EXTRA> constexpr int kDkvBlocks = DP * (int)sizeof(T) <= (EXTRA ? 192 : 256) ? 2 : 1;
template <class T, int DP, bool EXTRA> constexpr int kDkvFit = sizeof(T) == 4 && DP == 64 ? 2 : kDkvBlocks<T, DP, EXTRA>;

template <class T, int DP, bool VEC, bool EXTRA, bool HALF, int KS>
__global__ __launch_bounds__(AT_TPB, (kDkvBlocks<T, DP, EXTRA>)) void k_attention_dkv(AttnArgs p)
{
    constexpr int R = kDkvRows<DP, EXTRA, HALF, KS>, ROWS = AT_ROWS / KS;
    typedef AtTile<T, DP, R> Tile;
    typedef std::conditional_t<HALF, half_t, T> S;       // queries and keys
    typedef AtTile<S, DP, R> STile;
    constexpr int HALVES = kDkvHalves<T, DP, HALF>, ND = DP / 32 / HALVES, SUBS = Tile::ROWS / 32;
    static_assert(Tile::ROWS <= kAttnTile && kAttnTile % Tile::ROWS == 0, "");
    extern __shared__ __align__(256) unsigned char smem[];
    __shared__ int2 block_range[AT_WAVES];
    __shared__ int block_seen[AT_WAVES];
    const AttnShape &s = p.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ks = wave % KS;
    const int d = s.d, stride = s.stride(), per = s.heads / s.groups, ostride = s.heads * d;
    const AtBlock b = at_block(s);
    const int half = b.rest % HALVES, split = b.rest / HALVES % p.splits, key0 = at_key_block<KS>(p, b.n, b.rest / HALVES / p.splits) * ROWS;
    const int wave0 = key0 + 32 * (wave / KS), own = wave0 + (lane & 31);
    const int sstride = HALF ? (s.heads + s.groups) * d : stride;
    const S *base = (const S *)(HALF ? p.half : p.qk) + (size_t)b.n * s.T * sstride;

    // tiles of queries, from the first that sees one of the block's keys to the last
    const int all_tiles = (s.T + Tile::ROWS - 1) / Tile::ROWS;
    int first = 0, end = all_tiles, seen = s.T;                    // seen: end of the keys that some position sees
    const int4 *bounds = p.bounds + (size_t)b.n * 2 * ((s.T + kAttnTile - 1) / kAttnTile);
    if (s.mask == ATTN_CAUSAL) first = key0 / Tile::ROWS;
    if (s.mask == ATTN_SPANS) {
        first = all_tiles;
        end = seen = 0;
        for (int i = tid; i < all_tiles; i += AT_TPB) {
            const int4 v = bounds[i * Tile::ROWS / kAttnTile * 2];
            seen = max(seen, v.y);
            if (v.x < key0 + ROWS && v.y > key0) {
                first = min(first, i);
                end = i + 1;
            }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            first = min(first, __shfl_xor(first, o, 64));
            end = max(end, __shfl_xor(end, o, 64));
            seen = max(seen, __shfl_xor(seen, o, 64));
        }
        if (lane == 0) {
            block_range[wave] = {first, end};
            block_seen[wave] = seen;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) {
            first = min(first, block_range[w].x);
            end = max(end, block_range[w].y);
            seen = max(seen, block_seen[w]);
        }
    }
    first = __builtin_amdgcn_readfirstlane(first);
    end = __builtin_amdgcn_readfirstlane(end);
    // as with the queries, what is behind the last key that is seen is not read
    chunk16 key[Tile::STEPS], value[Tile::STEPS];
    at_own<S, DP, VEC>(key, own < seen ? base + (size_t)own * sstride + (size_t)(s.heads + b.g) * d : nullptr, d, lane);
    at_own<T, DP, VEC>(value, own < seen ? (const T *)p.v + ((size_t)b.n * s.T + own) * stride + (size_t)(s.heads + s.groups + b.g) * d : nullptr, d, lane);
    const float own_scale = HALF && own < seen ? p.half_scale[((size_t)(s.heads + b.g) * s.N + b.n) * s.T + own] : 1.0f;
    const int of_head = end > first ? end - first : 0, total = of_head * per;
    const int begin = (int)((long long)total * split / p.splits), stop = (int)((long long)total * (split + 1) / p.splits);

    const unsigned lds = at_lds(smem);
    AtStream<S, DP, VEC, R> queries(sstride, tid);
    AtStream<T, DP, VEC, R> gradients(ostride, tid);
    // of the rows of a tile, twice: 64 words each of lse, dout . o and scale, 128 of spans
    constexpr int ROW_BYTES = 5 * 256;
    constexpr int ROWS_AT = 4 * Tile::BYTES;
    // Head and tile of the loads that are under way, counted, so that addresses stay scalar.  Last tile first: with a causal mask all blocks of
    // a key head read the last ones.
    int next_head = 0, next_tile = 0;
    if (begin < stop) {
        next_head = __builtin_amdgcn_readfirstlane(b.g * per + begin / of_head);
        next_tile = __builtin_amdgcn_readfirstlane(end - 1 - begin % of_head);
    }
    auto fill = [&](int it) {
        const int head = next_head, q0 = next_tile * Tile::ROWS;
        // queries behind the last that sees something are not there: what padding holds is not read
        int there = s.T - q0;
        if (s.mask == ATTN_SPANS) there = min(there, bounds[q0 / kAttnTile * 2 + 1].x - q0 % kAttnTile);
        const unsigned row = lds + ROWS_AT + (it & 1) * ROW_BYTES;
        const size_t at = ((size_t)b.n * s.heads + head) * s.T + q0;
        if (wave == 0) at_dma4(p.lse + at, s.T - q0, row, tid);
        if (wave == 1) at_dma4(p.dsum + at, s.T - q0, row + 256, tid);
        if (HALF && wave == 2) at_dma4(p.half_scale + ((size_t)head * s.N + b.n) * s.T + q0, s.T - q0, row + 512, tid);
        if (s.mask == ATTN_SPANS && wave == 3) {
            const int2 *span = p.spans + (size_t)b.n * s.T + q0;
            at_dma4(span, 2 * (s.T - q0), row + 768, tid);
            at_dma4(span + 32, 2 * (s.T - q0) - 64, row + 1024, tid);
        }
        const int to = (it & 1) * 2 * Tile::BYTES;
        queries.fill(smem, lds, to, base + (size_t)q0 * sstride + (size_t)head * d, there, sstride, d, tid);
        gradients.fill(smem, lds, to + Tile::BYTES, (const T *)p.dout + ((size_t)b.n * s.T + q0) * ostride + (size_t)head * d, there, ostride, d, tid);
    };
    f32x16_t dk[ND] = {}, dv[ND] = {};
    float mult = HALF ? kAtRoom : 1.0f;
    AtScore score = {};
    int head_of = -1;
    if (begin < stop) fill(begin);
    for (int it = begin; it < stop; ++it) {
        const int at = it & 1;
        WAIT_VMCNT(0);
        at_barrier();
        const int head = next_head, q0 = next_tile * Tile::ROWS;
        if (head != head_of) score = at_score(s, head_of = head);
        if (--next_tile < first) {
            next_tile = end - 1;
            ++next_head;
        }
        if (it + 1 < stop) fill(it + 1);
        // what the tile's queries see, and whether all of them see all of the wave's keys
        bool none = wave0 >= s.T, whole = q0 + Tile::ROWS <= s.T;
        if (s.mask == ATTN_CAUSAL) {
            none |= q0 + Tile::ROWS <= wave0;
            whole &= q0 >= wave0 + 31;
        } else if (s.mask == ATTN_SPANS) {
            const int4 v = bounds[q0 / kAttnTile * 2];
            none |= v.x >= wave0 + 32 || v.y <= wave0;
            whole &= v.z <= wave0 && v.w >= wave0 + 32;
        }
        if (none) continue;
        const unsigned char *query = smem + at * 2 * Tile::BYTES, *dout = query + Tile::BYTES;
#pragma unroll 1
        for (int u = ks; u < SUBS; u += KS) {
            __builtin_amdgcn_sched_barrier(0);
            const int lane = at_again(tid) & 63, h = lane >> 5, k = wave0 + (lane & 31);
            const int r = 32 * u + 4 * h;                                // rows of a register's four: r + 8 g
            const unsigned char *row = smem + ROWS_AT + at * ROW_BYTES + 4 * r;
            const float by = score.scale * own_scale, unit = EXTRA ? 1.0f : by;
            float x[16], slope[16];
            f32x16_t w, dw;
            at_rows<S, STile>(w, query, 32 * u, key, d, lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = w[i];
            if (HALF)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 scale = *(const float4 *)(row + 512 + 32 * g);
                    x[4 * g] *= scale.x; x[4 * g + 1] *= scale.y; x[4 * g + 2] *= scale.z; x[4 * g + 3] *= scale.w;
                }
            if (EXTRA) at_bend<T, true>(x, score, by, (float)(k - (q0 + r)), slope);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 lse = *(const float4 *)(row + 32 * g);
                const float less[4] = {lse.x, lse.y, lse.z, lse.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * g + j] = __builtin_amdgcn_exp2f(fmaf(x[4 * g + j], unit, -less[j]));
            }
            if (!whole) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    int f[4] = {0, 0, 0, 0}, e[4];
                    if (s.mask == ATTN_SPANS) {
                        const int4 lo = *(const int4 *)(row + 768 + 4 * r + 64 * g), hi = *(const int4 *)(row + 768 + 4 * r + 64 * g + 16);
                        f[0] = lo.x; e[0] = lo.y; f[1] = lo.z; e[1] = lo.w;
                        f[2] = hi.x; e[2] = hi.y; f[3] = hi.z; e[3] = hi.w;
                    } else
#pragma unroll
                        for (int j = 0; j < 4; ++j) e[j] = s.mask == ATTN_CAUSAL ? q0 + r + 8 * g + j + 1 : s.T;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[4 * g + j] = k >= f[j] && k < e[j] ? x[4 * g + j] : 0.0f;
                }
            }
            at_columns<T, Tile>(dv, dout, 32 * u, half * ND, AtWeights<T>(x), d, lane);
            at_rows<T, Tile>(dw, dout, 32 * u, value, d, lane);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 dsum = *(const float4 *)(row + 256 + 32 * g);
                const float less[4] = {dsum.x, dsum.y, dsum.z, dsum.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[4 * g + j] *= dw[4 * g + j] - less[j];
                    if (EXTRA) x[4 * g + j] *= slope[4 * g + j];
                }
            }
            if (HALF) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 scale = *(const float4 *)(row + 512 + 32 * g);
                    x[4 * g] *= scale.x; x[4 * g + 1] *= scale.y; x[4 * g + 2] *= scale.z; x[4 * g + 3] *= scale.w;
                }
                at_fit(x, mult, dk);
            }
            at_columns<S, STile>(dk, query, 32 * u, half * ND, AtWeights<S>(x), d, lane);
        }
    }
    unsigned char *mine = smem + wave * kAtOwn<DP>;
    float by_mult = s.scale / mult;
    if constexpr (KS == 2) {
        float *theirs = (float *)(smem + wave / 2 * (64 * 32 * ND * 4));
        mine = (unsigned char *)theirs;
        at_barrier();                                      // the tiles are read
        if (ks) {
            at_give(theirs, dk, by_mult, lane);
            at_give(theirs + 64 * 16 * ND, dv, 1.0f, lane);
        }
        at_barrier();
        if (ks) return;
        at_take(theirs, dk, by_mult, 1.0f, lane);
        at_take(theirs + 64 * 16 * ND, dv, 1.0f, 1.0f, lane);
        by_mult = 1.0f;
    }
    if constexpr (VEC && sizeof(T) == 2 && HALVES == 1) {
        if (p.splits == 1) {
            if (KS == 1) at_barrier();                     // the tiles are read
            const size_t at_k = ((size_t)b.n * s.T + wave0) * stride + (size_t)(s.heads + b.g) * d;
            if (!p.dqk_float) at_store_rows<DP, ND>(mine, (T *)p.dqk + at_k, nullptr, stride, s.T - wave0, d, dk, by_mult, lane);
            else if (own < s.T)
                at_store<float, VEC, ND>(p.dqk_float + (((size_t)b.n * s.T + own) * (s.heads + s.groups) + s.heads + b.g) * d, d, 0, dk, by_mult, lane);
            at_store_rows<DP, ND>(mine, (T *)p.dv + at_k + (size_t)s.groups * d, nullptr, stride, s.T - wave0, d, dv, 1.0f, lane);
            return;
        }
    }
    if (own >= s.T) return;
    if (p.splits > 1) {
        float *to = p.part + ((((size_t)split * s.N + b.n) * s.groups + b.g) * s.T + own) * 2 * d;
        at_store<float, VEC, ND>(to, d, half * ND, dk, by_mult, lane);
        at_store<float, VEC, ND>(to + d, d, half * ND, dv, 1.0f, lane);
        return;
    }
    const size_t row = (size_t)b.n * s.T + own, at_k = row * stride + (size_t)(s.heads + b.g) * d;
    if (p.dqk_float) at_store<float, VEC, ND>(p.dqk_float + row * (s.heads + s.groups) * d + (size_t)(s.heads + b.g) * d, d, half * ND, dk, by_mult, lane);
    else at_store<T, VEC, ND>((T *)p.dqk + at_k, d, half * ND, dk, by_mult, lane);
    at_store<T, VEC, ND>((T *)p.dv + at_k + (size_t)s.groups * d, d, half * ND, dv, 1.0f, lane);
}

// The sums of all splits, V channels a thread (d a multiple of V, dqk and dv aligned to V elements)
template <class T, int V> __global__ __launch_bounds__(256) void k_attention_join(AttnArgs p)
{
    typedef vec_t<float, V> vecf;
    const AttnShape &s = p.s;
    const unsigned per = (unsigned)s.d / V, n = (unsigned)((size_t)s.N * s.groups * s.T * 2 * per), i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const unsigned half_row = i / per, e = (i - half_row * per) * V, row = half_row / 2;         // row: [N][groups][T]
    vecf sum = {};
#pragma unroll 4
    for (int k = 0; k < p.splits; ++k) {
        const vecf v = *(const vecf *)(p.part + ((size_t)k * n + i) * V);
#pragma unroll
        for (int j = 0; j < V; ++j) sum.e[j] += v.e[j];
    }
    const unsigned ng = row / (unsigned)s.T, t = row - ng * s.T, b = ng / (unsigned)s.groups, g = ng - b * s.groups;
    const size_t position = (size_t)b * s.T + t, at = position * s.stride() + (size_t)(s.heads + g) * s.d + e;
    if (!(half_row & 1) && p.dqk_float) {
        *(vecf *)(p.dqk_float + (position * (s.heads + s.groups) + s.heads + g) * s.d + e) = sum;
        return;
    }
    vec_t<T, V> out;
#pragma unroll
    for (int j = 0; j < V; ++j) out.e[j] = from_f32<T>(sum.e[j]);
    *(vec_t<T, V> *)(half_row & 1 ? (T *)p.dv + at + (size_t)s.groups * s.d : (T *)p.dqk + at) = out;
}

long long key_blocks(const AttnShape &s) { return (long long)s.N * s.groups * ((s.T + AT_ROWS - 1) / AT_ROWS); }

template <class T, int DP, bool VEC, bool EXTRA, bool HALF> struct Keys {
    template <int KS> static hipError_t launch(const AttnArgs &a, hipStream_t stream)
    {
        constexpr int smem = std::max(4 * AtTile<T, DP, kDkvRows<DP, EXTRA, HALF, KS>>::BYTES + 2 * 5 * 256, sizeof(T) == 2 ? AT_WAVES * kAtOwn<DP> : 0);
        return at_launch(k_attention_dkv<T, DP, VEC, EXTRA, HALF, KS>,
                         a.s.N * a.s.groups * ((a.s.T + AT_ROWS / KS - 1) / (AT_ROWS / KS)) * a.splits * kDkvHalves<T, DP, HALF>, smem, a, stream);
    }
    static hipError_t go(const AttnArgs &a, hipStream_t stream)
    {
        if constexpr (kAtShares<T, DP>)
            if (at_shares(a, key_blocks(a.s) * a.splits * kDkvHalves<T, DP, HALF>, kDkvFit<T, DP, EXTRA>)) return launch<2>(a, stream);
        return launch<1>(a, stream);
    }
};

// In how many parts the queries of the keys' sums are taken.  A block owns 128 keys of a key head, for all query heads that share it: few of
// them leave units idle or, where keys are seen by different numbers of queries, waiting for the longest.  Splits cost a pass over their sums:
// 12 heads of 80, 3 x 1003 positions without a mask, 288 blocks of the 512 that fit, us: 69 in one part, 59 and 14 in three.
// What fits is by the kernel that runs.  With two blocks a unit for all of up to 128 channels, a column's halves not counted, 16 / 4 heads of
// 128 with slopes over 2048 positions, causal, took 214 us a mini-batch, 184 so; 8 / 4 of 256 behind a ROTARY over 2 x 2048, causal, 482 and 454.
template <class T, int DP, bool VEC, bool EXTRA, bool HALF> struct Splits {
    static hipError_t go(const AttnArgs &a, int *out)
    {
        const AttnShape &s = a.s;
        const long long fit = (long long)a.units * kDkvFit<T, DP, EXTRA>, blocks = key_blocks(s) * kDkvHalves<T, DP, HALF>;
        const long long tiles = (long long)((s.T + 63) / 64) * (s.heads / s.groups);           // of queries
        long long splits = s.mask == ATTN_NONE ? fit / blocks : (2 * fit + blocks / 2) / blocks;
        if (splits > tiles / 4) splits = tiles / 4;
        *out = splits > 16 ? 16 : splits > 1 ? (int)splits : 1;
        return hipSuccess;
    }
};
int key_splits(int dt, AttnArgs a, int compute_units)
{
    a.units = compute_units > 0 ? compute_units : 256;
    int splits = 1;
    (void)at_dispatch<Splits>(dt, a, &splits);
    return splits;
}

}  // namespace

hipError_t attention_dkv(int dt, const AttnArgs &a, hipStream_t s)
{
    const hipError_t e = at_dispatch<Keys>(dt, a, s);
    if (e != hipSuccess || a.splits == 1) return e;
    // bf16 heads that are read element by element may be stored to a caller's dx that is aligned to one of them
    const bool vec = a.s.d % 4 == 0 && ((uintptr_t)a.dqk | (uintptr_t)a.dv) % (4 * dt_size(dt)) == 0;
    const size_t n = (size_t)a.s.N * a.s.groups * a.s.T * 2 * a.s.d / (vec ? 4 : 1);
    const dim3 grid((unsigned)((n + 255) / 256));
    if (dt == DT_F32 && vec) hipLaunchKernelGGL((k_attention_join<float, 4>), grid, dim3(256), 0, s, a);
    else if (dt == DT_F32) hipLaunchKernelGGL((k_attention_join<float, 1>), grid, dim3(256), 0, s, a);
    else if (vec) hipLaunchKernelGGL((k_attention_join<bf16_t, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attention_join<bf16_t, 1>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t attention_workspace(int dt, const AttnShape &a, bool half, int compute_units)
{
    AttnArgs q = {};
    q.s = a;
    if (half) q.half = &q;                                   // not read
    const int splits = key_splits(dt, q, compute_units);
    const size_t rows = ((size_t)a.N * a.heads * a.T * sizeof(float) + 255) / 256 * 256;
    return rows + (splits > 1 ? (size_t)splits * a.N * a.groups * a.T * 2 * a.d * sizeof(float) : 0);
}

hipError_t attention_bwd(int dt, AttnArgs a, void *workspace, int compute_units, hipStream_t s)
{
    a.dsum = (float *)workspace;
    a.part = (float *)((char *)workspace + ((size_t)a.s.N * a.s.heads * a.s.T * sizeof(float) + 255) / 256 * 256);
    a.splits = key_splits(dt, a, compute_units);
    const hipError_t e = attention_dq(dt, a, s);
    return e == hipSuccess ? attention_dkv(dt, a, s) : e;
}

}  // namespace bapipe
