// Attention, forward: o = softmax(scores) v in one pass over the keys, with a running maximum and sum per query.
// 4 x 4096 positions, causal, 32 / 8 heads of 128, bf16: 645 us, 852 TFLOP/s of the two products, of which 75 us are the second places for input
// and output.  The card runs at 1.7 to 1.8 GHz there; matrix instructions take 51 % of the cycles, and 64 keys of a wave 32 of them (1024
// cycles), 140 vector instructions and 32 exponentials.  No one of these bounds it: in an earlier form that took 711 us, leaving out the
// exponentials saved 5 %, LDS reads 6, loads of tiles and LDS reads 20, all three 27.
#include "attention_common.h"

namespace bapipe {
namespace {

// Rows of a tile.  With 32 keys at a time registers and LDS hold three blocks of heads of 128 channels a unit instead of two, and two of 192 and 256
// instead of one.  us with 64 and 32, while rows were still stored from the registers: 4 x 4096 positions, causal, 32 / 8 heads of 128: 705, 674;
// packed documents 173, 178; 4 x 2048, causal, 16 / 2 heads of 16-bit floats: 112, 101; 16 / 8 heads of 256: 295, 217, but with capped scores,
// which leave no registers for two, 192, 198.
template <class T, int DP, bool EXTRA, int KS>
constexpr int kFwdRows = KS == 1 && sizeof(T) == 2 && (DP == 128 || DP == 192 || (DP == 256 && !EXTRA)) ? 32 : 0;
template <class T, int DP, bool EXTRA, int KS>
constexpr int kFwdBlocks = sizeof(T) == 4 ? DP <= 64 ? 2 : 1 : KS == 1 && DP == 128 && !EXTRA ? 3 : DP <= 192 || kFwdRows<T, DP, EXTRA, KS> ? 2 : 1;

template <class T, int DP, bool VEC, bool EXTRA, bool HALF, int KS>
__global__ __launch_bounds__(AT_TPB, (kFwdBlocks<T, DP, EXTRA, KS>)) void k_attention_fwd(AttnArgs p)
{
    constexpr int R = kFwdRows<T, DP, EXTRA, KS>, ROWS = AT_ROWS / KS;
    typedef AtTile<T, DP, R> Tile;
    typedef std::conditional_t<HALF, half_t, T> S;       // what scores are made of
    typedef AtTile<S, DP, R> STile;
    constexpr int ND = DP / 32, SUBS = Tile::ROWS / 32 / KS;      // a wave's pieces of a tile: the KS u + ks-th
    extern __shared__ __align__(256) unsigned char smem[];
    __shared__ int2 block_range[AT_WAVES];
    const AttnShape &s = p.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, ks = wave % KS;
    const int d = s.d, stride = s.stride(), per = s.heads / s.groups;
    const AtBlock b = at_block(s);
    const int head = b.g * per + b.rest % per, q0 = at_query_block<KS>(p, b.n, b.rest / per) * ROWS;
    const int q = q0 + 32 * (wave / KS) + (lane & 31);
    const int sstride = HALF ? (s.heads + s.groups) * d : stride;
    const S *base = (const S *)(HALF ? p.half : p.qk) + (size_t)b.n * s.T * sstride, *keys = base + (size_t)(s.heads + b.g) * d;
    const T *values = (const T *)p.v + (size_t)b.n * s.T * stride + (size_t)(s.heads + s.groups + b.g) * d;
    const float *key_scale = HALF ? p.half_scale + ((size_t)(s.heads + b.g) * s.N + b.n) * s.T : nullptr;

    chunk16 query[Tile::STEPS];
    at_own<S, DP, VEC>(query, q < s.T ? base + (size_t)q * sstride + (size_t)head * d : nullptr, d, lane);
    if constexpr (VEC && !HALF) {
        if (p.copy) {                                      // its own queries and, for the first of their heads, the keys and values at their positions
            T *copy = (T *)p.copy + (size_t)b.n * s.T * stride;
#pragma unroll
            for (int c = 0; c < Tile::STEPS; ++c) {
                const int e = (2 * c + h) * Tile::EPC;
                if (ks == 0 && q < s.T && e < d) *(chunk16 *)(copy + (size_t)q * stride + (size_t)head * d + e) = query[c];
            }
            const int chunks = d / Tile::EPC, rows = min(ROWS, s.T - q0);
            for (int i = tid; head % per == 0 && i < 2 * rows * chunks; i += AT_TPB) {
                const int which = i / (rows * chunks), row = (i - which * rows * chunks) / chunks, chunk = i % chunks;
                const size_t at = (size_t)(q0 + row) * stride + (size_t)(s.heads + which * s.groups + b.g) * d + chunk * Tile::EPC;
                *(chunk16 *)(copy + at) = *(const chunk16 *)((const T *)p.qk + (size_t)b.n * s.T * stride + at);
            }
        }
    }
    const int2 span = at_span(p, b.n, q);
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
    if (HALF && q < s.T) by *= p.half_scale[((size_t)head * s.N + b.n) * s.T + q];
    const unsigned lds = at_lds(smem);
    AtStream<S, DP, VEC, R, false> key_stream(sstride, tid);
    AtStream<T, DP, VEC, R, false> value_stream(stride, tid);
    constexpr int SCALE_AT = 2 * 2 * Tile::BYTES;      // 64 words, twice
    auto fill = [&](int it) {
        const int k0 = first + it * Tile::ROWS;
        const int to = (it & 1) * 2 * Tile::BYTES;
        if (HALF && wave == 0) at_dma4(key_scale + k0, end - k0, lds + SCALE_AT + (it & 1) * 256, tid);
        key_stream.fill(smem, lds, to, keys + (size_t)k0 * sstride, end - k0, sstride, d, tid);
        value_stream.fill(smem, lds, to + Tile::BYTES, values + (size_t)k0 * stride, end - k0, stride, d, tid);
    };
    f32x16_t out[ND] = {};
    float top = -__builtin_inff(), sum = 0.0f;            // sum: of this half's keys
    const int tiles = (end - first + Tile::ROWS - 1) / Tile::ROWS;        // none where nobody sees anything
    if (tiles > 0) fill(0);
    for (int it = 0; it < tiles; ++it) {
        WAIT_VMCNT(0);
        at_barrier();                                      // the tile has arrived, the other one is read
        if (it + 1 < tiles) fill(it + 1);
        const int k0 = first + it * Tile::ROWS;
        if (k0 >= range.any.y || k0 + Tile::ROWS <= range.any.x) continue;
        const unsigned char *key = smem + (it & 1) * 2 * Tile::BYTES, *value = key + Tile::BYTES;
        float x[SUBS][16];
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
            f32x16_t w;
            at_rows<S, STile>(w, key, 32 * (KS * u + ks), query, d, lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[u][i] = w[i];
            if (HALF)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 r = *(const float4 *)(smem + SCALE_AT + (it & 1) * 256 + 4 * (32 * (KS * u + ks) + 8 * g + 4 * h));
                    x[u][4 * g] *= r.x; x[u][4 * g + 1] *= r.y; x[u][4 * g + 2] *= r.z; x[u][4 * g + 3] *= r.w;
                }
        }
        if (sizeof(T) == 2) at_order<SUBS * Tile::STEPS, 4>();
        if (EXTRA)
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                float none[16];
                at_bend<T, false>(x[u], score, by, (float)(q - (k0 + 32 * (KS * u + ks) + 4 * h)), none);
            }
        if (!(k0 >= range.all.x && k0 + Tile::ROWS <= range.all.y)) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = k0 + 32 * (KS * u + ks) + 8 * (i >> 2) + 4 * h + (i & 3);
                    x[u][i] = k >= span.x && k < span.y ? x[u][i] : -__builtin_inff();
                }
        }
        const float unit = EXTRA ? 1.0f : by;
        float most = x[0][0];
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, x[u][i]);
        most = at_halves_max(most) * unit;
        // The maximum that scores are taken relative to follows the true one only where that is 2^8 above: the sums stay far inside a float's
        // range, and most tiles leave the accumulators alone.
        if (__any(most > top + 8.0f)) {
            const float next = fmaxf(top, most), fade = next > -__builtin_inff() ? __builtin_amdgcn_exp2f(top - next) : 1.0f;
            top = next;
            sum *= fade;
#pragma unroll
            for (int t = 0; t < ND; ++t) out[t] *= fade;
        }
        const float less = top > -__builtin_inff() ? top : 0.0f;
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[u][i] = __builtin_amdgcn_exp2f(fmaf(x[u][i], unit, -less));
                sum += x[u][i];
            }
            at_columns<T, Tile>(out, value, 32 * (KS * u + ks), 0, AtWeights<T>(x[u]), d, lane);
        }
    }
    if (KS == 1) sum = at_halves_sum(sum);
    unsigned char *own = smem + wave * kAtOwn<DP>;
    if constexpr (KS == 2) {
        float *theirs = (float *)(smem + wave / 2 * (64 * (16 * ND + 2) * 4));
        own = (unsigned char *)theirs;
        at_barrier();                                      // the tiles are read
        if (ks) {
            at_give(theirs, out, 1.0f, lane);
            theirs[16 * ND * 64 + lane] = top;
            theirs[(16 * ND + 1) * 64 + lane] = sum;
        }
        at_barrier();
        if (ks) return;
        const float their_top = theirs[16 * ND * 64 + lane], both = fmaxf(top, their_top);
        const float mine = top > -__builtin_inff() ? __builtin_amdgcn_exp2f(top - both) : 0.0f;
        const float other = their_top > -__builtin_inff() ? __builtin_amdgcn_exp2f(their_top - both) : 0.0f;
        at_take(theirs, out, mine, other, lane);
        sum = sum * mine + theirs[(16 * ND + 1) * 64 + lane] * other;
        top = both;
        sum = at_halves_sum(sum);
    }
    const bool sees = span.x < span.y;
    const float by_sum = sees ? 1.0f / sum : 0.0f;
    if constexpr (VEC && sizeof(T) == 2) {
        if (KS == 1) at_barrier();                         // the tiles are read
        const int row0 = q0 + 32 * (wave / KS), rows = s.T - row0;
        const size_t at_o = ((size_t)b.n * s.T + row0) * s.heads * d + (size_t)head * d, ostride = (size_t)s.heads * d;
        at_store_rows<DP, ND>(own, (T *)p.o + at_o, p.o2 ? (T *)p.o2 + at_o : nullptr, ostride, rows, d, out, by_sum, lane);
        at_store_low_rows<DP, ND>(own, p.o_low + at_o, ostride, rows, d, out, by_sum, lane);
    } else if (q < s.T) {
        const size_t at_o = ((size_t)b.n * s.T + q) * s.heads * d + (size_t)head * d;
        at_store<T, VEC, ND>((T *)p.o + at_o, d, 0, out, by_sum, lane);
        if (p.o2) at_store<T, VEC, ND>((T *)p.o2 + at_o, d, 0, out, by_sum, lane);
        if (sizeof(T) == 2) at_store_low<ND>(p.o_low + at_o, d, out, by_sum, lane);
    }
    if (q >= s.T) return;
    if (h == 0) p.lse[((size_t)b.n * s.heads + head) * s.T + q] = sees ? top + log2f(sum) : __builtin_inff();
}

template <class T, int DP, bool VEC, bool EXTRA, bool HALF> struct Forward {
    template <int KS> static hipError_t launch(const AttnArgs &a, hipStream_t stream)
    {
        constexpr int smem = std::max(4 * AtTile<T, DP, kFwdRows<T, DP, EXTRA, KS>>::BYTES + (HALF ? 512 : 0), sizeof(T) == 2 ? AT_WAVES * kAtOwn<DP> : 0);
        return at_launch(k_attention_fwd<T, DP, VEC, EXTRA, HALF, KS>, a.s.N * a.s.heads * ((a.s.T + AT_ROWS / KS - 1) / (AT_ROWS / KS)), smem, a, stream);
    }
    static hipError_t go(const AttnArgs &a, hipStream_t stream)
    {
        if constexpr (kAtShares<T, DP>)
            if (at_shares(a, (long long)a.s.N * a.s.heads * ((a.s.T + AT_ROWS - 1) / AT_ROWS))) return launch<2>(a, stream);
        return launch<1>(a, stream);
    }
};

// One wave to a tile of kAttnTile positions
__global__ __launch_bounds__(64) void k_attention_spans(const int32_t *given, int2 *spans, int4 *bounds, int T)
{
    const int lane = threadIdx.x, n = blockIdx.y, t = blockIdx.x * kAttnTile + lane;
    int4 b = {T, 0, 0, T};
    int count = 0;
    if (t < T) {
        const size_t at = (size_t)n * T + t;
        int2 v = given ? int2{max(given[2 * at], 0), min(given[2 * at + 1], T)} : int2{0, t + 1};
        if (v.x >= v.y) v = {0, 0};
        spans[at] = v;
        b = v.x < v.y ? int4{v.x, v.y, v.x, v.y} : int4{T, 0, T, 0};
        count = v.x < v.y ? lane + 1 : 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        b.x = min(b.x, __shfl_xor(b.x, o, 64));
        b.y = max(b.y, __shfl_xor(b.y, o, 64));
        b.z = max(b.z, __shfl_xor(b.z, o, 64));
        b.w = min(b.w, __shfl_xor(b.w, o, 64));
        count = max(count, __shfl_xor(count, o, 64));
    }
    if (lane == 0) {
        bounds[2 * ((size_t)n * gridDim.x + blockIdx.x)] = b;
        bounds[2 * ((size_t)n * gridDim.x + blockIdx.x) + 1] = {count, 0, 0, 0};
    }
}

// The blocks of a sample with the most to do first: the last ones to be started are what others wait for.  Documents of 1500 to 4500 in 16384
// positions, 8 heads of 128 that share one key head, 1024 blocks of which 512 fit, us for the three kernels: 206, 243 and 354 from the last
// position to the first, 170, 188 and 302 so, and 6 for this.
// Blocks of queries by the tiles from the first to the last key that one of them sees, blocks of keys by the tiles of queries that see one of them;
// a block's place is the number of those in front of it.
constexpr int kOrderBlocks = 1024;      // of more the others' work is long enough
__global__ __launch_bounds__(1024) void k_attention_order(const int4 *bounds, int *order, int T)
{
    constexpr int L = 8, SPT = 1024 / L;      // lanes to a block, which share its sums
    __shared__ int2 range[kOrderBlocks * AT_ROWS / kAttnTile];
    __shared__ int work[kOrderBlocks];
    const int tiles = (T + kAttnTile - 1) / kAttnTile, blocks = (T + AT_ROWS - 1) / AT_ROWS, part = threadIdx.x % L, which = blockIdx.y;
    bounds += (size_t)blockIdx.x * 2 * tiles;
    order += ((size_t)blockIdx.x * 2 + which) * blocks;
    for (int i = threadIdx.x; i < tiles; i += 1024) range[i] = *(const int2 *)&bounds[2 * i];
    __syncthreads();
    auto sum = [&](int n) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
        return n;
    };
    for (int b0 = 0; b0 < blocks; b0 += SPT) {
        const int b = b0 + threadIdx.x / L;
        int n = 0;
        if (which == 0) {
            int first = T, end = 0;
            for (int i = b * (AT_ROWS / kAttnTile); i < (b + 1) * (AT_ROWS / kAttnTile) && i < tiles; ++i) {
                first = min(first, range[i].x);
                end = max(end, range[i].y);
            }
            n = max(end - first, 0) / kAttnTile;
        } else {
#pragma unroll 4
            for (int i = part; i < tiles; i += L) n += range[i].x < (b + 1) * AT_ROWS && range[i].y > b * AT_ROWS;
            n = sum(n);
        }
        if (part == 0 && b < blocks) work[b] = n;
    }
    __syncthreads();
    for (int b0 = 0; b0 < blocks; b0 += SPT) {
        const int b = b0 + threadIdx.x / L, mine = b < blocks ? work[b] : 0;
        int place = 0;
#pragma unroll 4
        for (int i = part; i < blocks; i += L) place += work[i] > mine || (work[i] == mine && i < b);
        place = sum(place);
        if (part == 0 && b < blocks) order[place] = b;
    }
}

}  // namespace

// Sequences of less than eight blocks are over too soon
size_t attention_order_size(int N, int T)
{
    const int blocks = (T + AT_ROWS - 1) / AT_ROWS;
    return blocks >= 8 && blocks <= kOrderBlocks ? (size_t)N * 2 * blocks : 0;
}

hipError_t attention_spans(const int32_t *given, int2 *spans, int4 *bounds, int *order, int N, int T, hipStream_t s)
{
    // a sample's tiles are a row of the grid, which takes 65535 of them at a time
    const int tiles = (T + kAttnTile - 1) / kAttnTile;
    for (int n = 0; n < N; n += 65535) {
        const size_t at = (size_t)n * T;
        hipLaunchKernelGGL(k_attention_spans, dim3((unsigned)tiles, (unsigned)(N - n < 65535 ? N - n : 65535)), dim3(64), 0, s, given ? given + 2 * at : nullptr,
                           spans + at, bounds + (size_t)n * 2 * tiles, T);
    }
    if (order) hipLaunchKernelGGL(k_attention_order, dim3((unsigned)N, 2), dim3(1024), 0, s, (const int4 *)bounds, order, T);
    return hipGetLastError();
}

// A launch holds less than 2^32 threads.  Where blocks are many nothing makes more of them: two waves share 32 rows, and sums are split, where blocks
// are no more than a few times the units, and heads whose columns are taken in halves (of keys) are too wide for 2^23 of them in 2 GiB.
bool attention_launches(int N, int heads, int T) { return (long long)N * heads * ((T + AT_ROWS - 1) / AT_ROWS) < (1ll << 32) / AT_TPB; }

hipError_t attention_fwd(int dt, const AttnArgs &a, hipStream_t s) { return at_dispatch<Forward>(dt, a, s); }

}  // namespace bapipe
