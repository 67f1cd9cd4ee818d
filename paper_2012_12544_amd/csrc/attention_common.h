// Pieces shared by the attention kernels (kernels_attention_*.hip).
//
// One wave owns 32 rows of one axis (queries in the forward pass and for dq, keys for dk and dv), one to a lane of either half, whose
// values stay in registers as the right operand of the 32x32 MFMAs; the other axis streams through LDS in tiles.  With streamed rows
// as the left operand a product of both comes out with the owned row in the lane and streamed rows in the registers:
//     register i of lane l: owned row l & 31, streamed row 8 (i / 4) + 4 (l / 32) + i % 4 of the tile's 32.
// Sums over streamed rows are sums over registers, with one exchange between the halves.  And the next product, which sums over the
// streamed rows, finds its right operand in those registers as they are: the order of a product's summands is free, so its left operand
// is read with the same order of rows (bf16: transposing LDS reads of four rows each; float: single words).
// Nothing of a score's size ever leaves the registers.
#pragma once
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "mfma_common.h"

namespace bapipe {

constexpr int AT_WAVES = 4, AT_TPB = 64 * AT_WAVES, AT_ROWS = 32 * AT_WAVES;      // rows that a block owns

// 16-bit floats, where bf16_t is the other type of that size
struct half_t {
    uint16_t v;
};

// A tile of rows of DP elements in LDS, in groups of 64 bytes of every row: group after group, each of all rows.  The four 16-byte chunks of a
// row in a group change places with the row / 4, so that both kinds of reads meet each bank once - 16 rows at one chunk (row operands),
// four rows at four chunks (transposing reads) - and everything but two lane addresses of either kind is an immediate offset.  (With whole
// rows one after the other and a chunk's place XORed with the row every step and column tile took an address register of its own,
// and the kernel for dk and dv spilled 106.)  Loads bring 64 bytes of 16 rows at a time.
// R: rows, 0 for what two operands, twice, in 128 KB leave
template <class T, int DP, int R = 0> struct AtTile {
    static constexpr int EPC = 16 / (int)sizeof(T);                   // elements of a chunk
    static constexpr int CH = DP / EPC, RB = DP * (int)sizeof(T);     // chunks, bytes of a row
    static constexpr int STEPS = CH / 2;                              // a step of a row product takes two chunks, one for each half
    static constexpr int ROWS = R ? R : RB <= 512 ? 64 : 32;
    static constexpr int BYTES = ROWS * RB;
    static __device__ __forceinline__ int at(int group, int row, int chunk) { return (group * ROWS + row) * 64 + ((chunk ^ ((row >> 2) & 3)) << 4); }
    // row and chunk of the i-th 16 bytes
    static __device__ __forceinline__ int row_of(int i) { return i / 4 % ROWS; }
    static __device__ __forceinline__ int chunk_of(int i) { return i / (4 * ROWS) * 4 + ((i & 3) ^ ((row_of(i) >> 2) & 3)); }
};

// acc += streamed rows x owned rows over one step of their elements
template <class T> __device__ __forceinline__ void at_mma(f32x16_t &acc, chunk16 a, chunk16 b)
{
    typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
    if constexpr (std::is_same<T, half_t>::value)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), acc, 0, 0, 0);
    else if constexpr (sizeof(T) == 2) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_frag(a), as_frag(b), acc, 0, 0, 0);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
}

// The order of N LDS reads and as many matrix instructions: AHEAD reads first, then one for every instruction
template <int N, int AHEAD> __device__ __forceinline__ void at_order()
{
    constexpr int first = AHEAD < N ? AHEAD : N;
    __builtin_amdgcn_sched_group_barrier(0x100, first, 0);
#pragma unroll
    for (int i = 0; i < N - first; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, first, 0);
}

// acc = 32 streamed rows from row0 of the tile x owned rows.  Floats leave out what is behind their d elements: their tiles are built for 64, 128
// and 256, and a step takes four instructions of 64 cycles.
template <class T, class Tile>
__device__ __forceinline__ void at_rows(f32x16_t &acc, const unsigned char *tile, int row0, const chunk16 (&own)[Tile::STEPS], int d, int lane)
{
    const int row = lane & 31, h = lane >> 5;
    acc = f32x16_t{};
#pragma unroll
    for (int c = 0; c < Tile::STEPS; ++c)
        if (sizeof(T) == 2 || 2 * c * Tile::EPC < d)
            at_mma<T>(acc, *(const chunk16 *)(tile + Tile::at(0, row, 2 * (c & 1) + h) + ((c >> 1) * Tile::ROWS + row0) * 64), own[c]);
}

// The right operand of a product that sums over 32 streamed rows: the registers of at_rows, in the storage type
template <class T> struct AtWeights {
    float v[16];
    __device__ __forceinline__ explicit AtWeights(const float (&x)[16])
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = x[i];
    }
};
template <> struct AtWeights<bf16_t> {
    uint32_t v[8];
    __device__ __forceinline__ explicit AtWeights(const float (&x)[16])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
};
template <> struct AtWeights<half_t> {
    uint32_t v[8];
    __device__ __forceinline__ explicit AtWeights(const float (&x)[16])
    {
        typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), f16x2_t));
    }
};

// acc[t][element 32 (t0 + t) + register's row][owned row] += sum over the 32 streamed rows from row0 of their elements x weights
template <class T, class Tile, int ND>
__device__ __forceinline__ void at_columns(f32x16_t (&acc)[ND], const unsigned char *tile, int row0, int t0, const AtWeights<T> &w, int d, int lane)
{
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) s16x4_t lds_v4;
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const int sl = lane & 15, chunk = 2 * ((lane >> 4) & 1) + ((sl & 3) >> 1), row = 4 * h + (sl >> 2);
        const unsigned char *from = tile + t0 * (Tile::ROWS * 64);
        const int lo_at = Tile::at(0, row, chunk) + 8 * (sl & 1), hi_at = Tile::at(0, row + 8, chunk) + 8 * (sl & 1);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const chunk16 b = {w.v[4 * c], w.v[4 * c + 1], w.v[4 * c + 2], w.v[4 * c + 3]};
#pragma unroll
            for (int t = 0; t < ND; ++t) {
                const int off = (t * Tile::ROWS + row0 + 16 * c) * 64;
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(from + lo_at + off));
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(from + hi_at + off));
                const s16x8_t a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                at_mma<T>(acc[t], __builtin_bit_cast(chunk16, a), b);
            }
        }
    } else {
        const int e = lane & 31;
        const unsigned char *from = tile + 2 * t0 * (Tile::ROWS * 64);
#pragma unroll
        for (int t = 0; t < ND; ++t) {
            if (32 * (t0 + t) >= d) break;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = Tile::at(e >> 4, 8 * ((i >> 2) & 1) + 4 * h, (e >> 2) & 3) + 4 * (e & 3);
                const float a = *(const float *)(from + at + (2 * t * Tile::ROWS + row0 + 16 * (i >> 3) + (i & 3)) * 64);
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.v[i], acc[t], 0, 0, 0);
            }
        }
    }
}

// the other half's value of an owned row, combined with this one's
__device__ __forceinline__ float at_halves_max(float v) { return fmaxf(v, __shfl_xor(v, 32, 64)); }
__device__ __forceinline__ float at_halves_sum(float v) { return v + __shfl_xor(v, 32, 64); }

// 16-bit floats as weights: x times a power of two of the owned row's, mult, that takes the largest of all so far to at most 2^15 of a format that
// ends at 65504.  It falls where a larger one comes, by so much that the next few times larger fit too, and what was summed up follows; weights
// 2^25 below the largest lose digits, which are 2^-36 of the sum.  kAtRoom, the mult to begin with, takes all below 2^-85 as they are.
constexpr float kAtRoom = 0x1p100f;
template <int ND> __device__ __forceinline__ void at_fit(float (&x)[16], float &mult, f32x16_t (&acc)[ND])
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(x[i]));
    most = at_halves_max(most);
    const bool over = most * mult > 0x1p15f;
    if (__any(over)) {
        const float next = over ? fminf(ldexpf(1.0f, 11 - __builtin_amdgcn_frexp_expf(most)), kAtRoom) : mult, fade = next / mult;
        mult = next;
#pragma unroll
        for (int t = 0; t < ND; ++t) acc[t] *= fade;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= mult;
}

// The chunks of an owned row, which lies at `row` (NULL: zeros) with d elements
template <class T> __device__ __forceinline__ T at_zero()
{
    T z;
    __builtin_memset(&z, 0, sizeof z);
    return z;
}
template <class T, int DP, bool VEC> __device__ __forceinline__ void at_own(chunk16 *own, const T *row, int d, int lane)
{
    typedef AtTile<T, DP> Tile;
    constexpr int EPC = Tile::EPC;
#pragma unroll
    for (int c = 0; c < Tile::STEPS; ++c) {
        const int e0 = (2 * c + (lane >> 5)) * EPC;
        own[c] = chunk16{0, 0, 0, 0};
        if constexpr (VEC) {
            if (row && e0 < d) own[c] = *(const chunk16 *)(row + e0);
        } else {
            vec_t<T, EPC> v;
#pragma unroll
            for (int j = 0; j < EPC; ++j) v.e[j] = row && e0 + j < d ? row[e0 + j] : at_zero<T>();
            own[c] = __builtin_bit_cast(chunk16, v);
        }
    }
}

// dma16 of a resource that differs from tile to tile: it may have been written by a vector instruction (a lane read back from a spilled
// scalar) just before, which a load has to be five states behind of, and the compiler counts none inside of assembly
// OFF: more bytes of the address in memory; the instruction adds them to that in LDS too, from which they are taken off
template <int OFF> __device__ __forceinline__ void at_dma16(__amdgpu_buffer_rsrc_t rsrc, unsigned lds_addr, unsigned voffset)
{
    static_assert(OFF >= 0 && OFF < 4096, "");
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen offset:%3 lds" ::"s"(lds_addr - OFF), "v"(voffset), "s"(rsrc), "n"(OFF));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t at_resource(const void *from, int bytes)
{
    const uint64_t address = (uint64_t)(uintptr_t)from;
    const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)address), high = __builtin_amdgcn_readfirstlane((uint32_t)(address >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)(((uint64_t)high << 32) | low), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// v, of which the compiler does not know that it is the same every time: what is made of it in a loop is made there again, in a few instructions,
// and does not occupy registers all the while.  (A register that is spilled is read back behind all loads under way.)
__device__ __forceinline__ int at_again(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// 4 bytes a lane, of rows of a tile's: lane l's word lands at lds_addr + 4 l, zero from word `words` on
__device__ __forceinline__ void at_dma4(const void *from, int words, unsigned lds_addr, int tid)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds_addr), "v"((at_again(tid) & 63) * 4),
                 "s"(at_resource(from, words > 0 ? words * 4 : 0)));
}

template <int OFF> __device__ __forceinline__ void at_dma4(__amdgpu_buffer_rsrc_t rsrc, unsigned lds_addr, unsigned voffset)
{
    static_assert(OFF >= 0 && OFF < 4096, "");
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen offset:%3 lds" ::"s"(lds_addr - OFF), "v"(voffset), "s"(rsrc), "n"(OFF));
}

// Fills tiles from rows of d elements, `stride` elements apart.  VEC: d a multiple of a chunk and 16-byte aligned rows.  These and all floats, which
// come word by word, are asynchronous: complete after WAIT_VMCNT(0) and a barrier.
// (Causal float heads of 45 channels, 4 x 1024 positions, 8 of them, a mini-batch: 431 us element by element through registers, 356.)
// Rows that are not there, and what is behind d, are zeros: zero times zero is what the products see of them, whatever memory holds.
// AGAIN: a lane's place is worked out again for every tile (see at_again), else it is kept.
template <class T, int DP, bool VEC, int R = 0, bool AGAIN = true> struct AtStream {
    typedef AtTile<T, DP, R> Tile;
    // chunks of a row that the block loads at once, and how often
    static constexpr int TPB = AT_TPB, STEP = TPB / Tile::ROWS, ISSUES = Tile::ROWS * Tile::CH / TPB;
    static_assert(Tile::ROWS * Tile::CH % TPB == 0, "");
    int row = 0, chunk = 0;
    unsigned voff = 0;
    __device__ __forceinline__ AtStream(int stride, int tid)
    {
        static_assert(STEP % 4 == 0, "");
        if (VEC && !AGAIN) place(stride, tid);
    }
    __device__ __forceinline__ void place(int stride, int tid)
    {
        row = Tile::row_of(tid);
        chunk = Tile::chunk_of(tid);
        voff = (unsigned)row * (unsigned)(stride * (int)sizeof(T)) + chunk * 16;
    }
    template <int I> static __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rsrc, unsigned lds_addr, unsigned at, int chunk, int chunks)
    {
        if constexpr (I < ISSUES) {
            at_dma16<I * STEP * 16>(rsrc, lds_addr + I * TPB * 16, chunk < chunks - I * STEP ? at : 0x80000000u);
            issue<I + 1>(rsrc, lds_addr, at, chunk, chunks);
        }
    }
    // words of a group of 64 bytes: 16 rows at once
    template <int G> static __device__ __forceinline__ void words(__amdgpu_buffer_rsrc_t rsrc, unsigned lds_addr, unsigned at, int left)
    {
        if constexpr (G < DP / 16) {
            at_dma4<G * 64>(rsrc, lds_addr + G * Tile::ROWS * 64, 16 * G < left ? at : 0x80000000u);
            words<G + 1>(rsrc, lds_addr, at, left);
        }
    }
    // to: the tile's place in the block's LDS, which begins at `lds`; from: the tile's first row; rows: how many there are from it on
    __device__ __forceinline__ void fill(unsigned char *smem, unsigned lds, int to, const T *from, int rows, int stride, int d, int tid)
    {
        if constexpr (VEC) {
            const int n = rows < Tile::ROWS ? rows : Tile::ROWS;
            const int bytes = n > 0 ? (int)(((long long)(n - 1) * stride + d) * (int)sizeof(T)) : 0;
            const __amdgpu_buffer_rsrc_t rsrc = at_resource(from, bytes);
            if (AGAIN) place(stride, at_again(tid));
            const unsigned at = row < n ? voff : 0x80000000u;      // rows that are there lie within 2 GiB
            const unsigned lds_addr = lds + to + (unsigned)__builtin_amdgcn_readfirstlane(tid >> 6) * 1024;
            if (d == DP) issue<0>(rsrc, lds_addr, at, 0, 1 << 20);
            else issue<0>(rsrc, lds_addr, at, chunk, d / Tile::EPC);
        } else if constexpr (sizeof(T) == 4) {
            const int n = rows < Tile::ROWS ? rows : Tile::ROWS;
            const int bytes = n > 0 ? (int)(((long long)(n - 1) * stride + d) * 4) : 0;
            const __amdgpu_buffer_rsrc_t rsrc = at_resource(from, bytes);
            const int t = at_again(tid), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
            const int e = 4 * (((t >> 2) & 3) ^ wave) + (t & 3);                  // row / 4 of a lane's rows is the wave, modulo 4
#pragma unroll
            for (int q = 0; q < Tile::ROWS / 16; ++q) {
                const int r = 16 * q + (t >> 4);
                words<0>(rsrc, lds + to + q * 1024 + wave * 256, r < n ? (unsigned)r * (unsigned)(stride * 4) + 4 * e : 0x80000000u, d - e);
            }
        } else {
            constexpr int AT_ONCE = 32 / Tile::EPC < ISSUES ? 32 / Tile::EPC : ISSUES;      // 32 loads under way
            static_assert(ISSUES % AT_ONCE == 0, "");
#pragma unroll 1
            for (int i0 = 0; i0 < ISSUES; i0 += AT_ONCE) {
                vec_t<T, Tile::EPC> v[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    const int at = (i0 + i) * TPB + tid, row = Tile::row_of(at), e0 = Tile::chunk_of(at) * Tile::EPC;
#pragma unroll
                    for (int j = 0; j < Tile::EPC; ++j) v[i].e[j] = row < rows && e0 + j < d ? from[(size_t)row * stride + e0 + j] : at_zero<T>();
                }
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) *(chunk16 *)(smem + to + ((i0 + i) * TPB + tid) * 16) = __builtin_bit_cast(chunk16, v[i]);
            }
        }
    }
};

// What is done to a score on its way to the softmax, in units of log 2
constexpr float kLog2e = 1.44269504088896341f;
struct AtScore {
    float scale;         // log2(e) / sqrt(d)
    float cap, per_cap;  // log2(e) times the cap, and one over that; 0: none
    float fall;          // log2(e) times the head's slope; 0: no bias
};
__device__ __forceinline__ AtScore at_score(const AttnShape &a, int head)
{
    auto uniform = [](float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); };
    AtScore s;
    s.scale = a.scale * kLog2e;
    s.cap = uniform(a.cap * kLog2e);
    s.per_cap = a.cap > 0.0f ? 1.0f / s.cap : 0.0f;
    s.fall = uniform(a.bias ? kLog2e * exp2f(-(float)a.bias * (float)(head + 1) / (float)a.heads) : 0.0f);
    return s;
}
// Scores of at_rows to logarithms base 2, register i of a key (or query) 8 (i / 4) + i % 4 further on than the first; slope receives the
// derivative of the cap.  tanh x = 1 - 2 r with r = 1 / (1 + e^2x), whose derivative is 4 r (1 - r).  In a bf16 stage that is off by 2^-24 of the
// cap, which caps of up to 4096 can afford; above them, and in float stages, the function is called.
// The registers are taken out of the product one by one first: with elements of the vector changed behind branches the compiler has stored one
// of them over its neighbours where accumulators lie in AGPRs (float heads of 128, bf16 ones of 256 channels).
template <class T, bool SLOPE>
__device__ __forceinline__ void at_bend(float (&x)[16], const AtScore &p, float by, float distance, float (&slope)[16])
{
    if (SLOPE)
#pragma unroll
        for (int i = 0; i < 16; ++i) slope[i] = 1.0f;
    if (sizeof(T) == 2 && p.cap > 0.0f && p.cap < 4096.0f * kLog2e) {
        const float twice = by * p.per_cap * (2.0f * kLog2e);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * twice));
            x[i] = fmaf(-2.0f * p.cap, r, p.cap);
            if (SLOPE) slope[i] = 4.0f * r * (1.0f - r);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= by;
        if (p.cap > 0.0f)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float th = tanhf(x[i] * p.per_cap);
                x[i] = p.cap * th;
                if (SLOPE) slope[i] = 1.0f - th * th;
            }
    }
    if (p.fall != 0.0f)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] -= p.fall * fabsf(distance - (float)(8 * (i >> 2) + (i & 3)));
}

// keys that the query at t of sample n sees: [x, y), none where x >= y
__device__ __forceinline__ int2 at_span(const AttnArgs &a, int n, int t)
{
    if (t >= a.s.T) return {a.s.T, 0};
    if (a.s.mask == ATTN_NONE) return {0, a.s.T};
    if (a.s.mask == ATTN_CAUSAL) return {0, t + 1};
    const int2 v = a.spans[(size_t)n * a.s.T + t];
    return v.x < v.y ? v : int2{a.s.T, 0};
}

// What the 32 queries of a wave see: some of them [any.x, any.y), all of them [all.x, all.y)
struct AtRange {
    int2 any, all;
};
__device__ __forceinline__ AtRange at_wave_range(int2 span)
{
    AtRange r{span, span};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        r.any.x = min(r.any.x, __shfl_xor(r.any.x, o, 64));
        r.any.y = max(r.any.y, __shfl_xor(r.any.y, o, 64));
        r.all.x = max(r.all.x, __shfl_xor(r.all.x, o, 64));
        r.all.y = min(r.all.y, __shfl_xor(r.all.y, o, 64));
    }
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return {{uniform(r.any.x), uniform(r.any.y)}, {uniform(r.all.x), uniform(r.all.y)}};
}

// Block to (sample, key head) and the rest.  Samples and key heads change fastest: blocks go round the XCDs, so that where there are a
// multiple of eight of them the blocks that read the same keys share an L2.
struct AtBlock {
    int n, g, rest;
};
__device__ __forceinline__ AtBlock at_block(const AttnShape &s)
{
    const int of = s.N * s.groups, ng = blockIdx.x % of;
    return {ng / s.groups, ng % s.groups, (int)(blockIdx.x / of)};
}

// KS waves of a block share 32 rows, each for its part of every tile's 32-row pieces, and add up what they have in LDS at the end: where rows are
// few that makes twice as many blocks, or keeps waves busy that have no rows of their own.  Tiles of 64 rows.  us for the forward pass, dq and dkv
// with KS 1 and 2: 4 x 333 positions of 6 / 2 float heads of 45, 72 blocks of 128 rows: 40, 52, 67 and 28, 34, 43; 64 x 50 of 16 / 4 heads of 64:
// 14.2, 15.2, 14.6 and 13.9, 14.9, 12.2; but 3 x 1003 of 12 heads of 80, 288 blocks for 256 units: 49, 55, 66 and 45, 58, 73.  (One rule for all
// three: the forward pass by itself would share a little beyond it.)
template <class T, int DP> constexpr bool kAtShares = AtTile<T, DP>::ROWS == 64;
// per_unit: so many of the blocks, which are twice as many then, a unit holds at once; more than that take a second round.  dkv of wide heads,
// one block a unit, a mini-batch of 1003 positions without a mask, us: 12 heads of 192 172 in 384 blocks of KS 2, 130 in 192 of KS 1, the
// sums in two parts in both; 12 of 256 306 and 166 (KS 2 spills 264 registers there).
inline bool at_shares(const AttnArgs &a, long long blocks, int per_unit = 2) { return a.s.T <= 64 || 2 * blocks <= (long long)a.units * per_unit; }

// Which block of rows is the i-th to be started: those with the most to do first, with a causal mask the last queries and the first keys
template <int KS> __device__ __forceinline__ int at_query_block(const AttnArgs &a, int n, int i)
{
    const int blocks = (a.s.T + AT_ROWS / KS - 1) / (AT_ROWS / KS);
    return KS == 1 && a.order ? __builtin_amdgcn_readfirstlane(a.order[(size_t)n * 2 * blocks + i]) : blocks - 1 - i;
}
template <int KS> __device__ __forceinline__ int at_key_block(const AttnArgs &a, int n, int i)
{
    const int blocks = (a.s.T + AT_ROWS / KS - 1) / (AT_ROWS / KS);
    return KS == 1 && a.order ? __builtin_amdgcn_readfirstlane(a.order[((size_t)n * 2 + 1) * blocks + i]) : i;
}
// accumulators of a lane to its wave's partner and back, a float at a time in a row of all lanes
template <int ND> __device__ __forceinline__ void at_give(float *to, const f32x16_t (&acc)[ND], float by, int lane)
{
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) to[(16 * t + i) * 64 + lane] = acc[t][i] * by;
}
template <int ND> __device__ __forceinline__ void at_take(const float *from, f32x16_t (&acc)[ND], float mine, float theirs, int lane)
{
#pragma unroll
    for (int t = 0; t < ND; ++t) {
        f32x16_t v;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = from[(16 * t + i) * 64 + lane];
        acc[t] = acc[t] * mine + v * theirs;
    }
}

// address of the dynamic LDS
__device__ __forceinline__ unsigned at_lds(const unsigned char *smem) { return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_void_t *)smem); }

__device__ __forceinline__ void at_barrier()
{
    WAIT_LGKMCNT(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// four neighbouring elements of a row of d, from element e0 on
template <class T, bool VEC> __device__ __forceinline__ void at_store4(T *row, int e0, int d, float x0, float x1, float x2, float x3)
{
    vec_t<T, 4> v;
    if constexpr (sizeof(T) == 2) {
        const chunk8 c = {pack_bf16(x0, x1), pack_bf16(x2, x3)};
        v = __builtin_bit_cast(vec_t<T, 4>, c);
    } else {
        const chunk16 c = {__float_as_uint(x0), __float_as_uint(x1), __float_as_uint(x2), __float_as_uint(x3)};
        v = __builtin_bit_cast(vec_t<T, 4>, c);
    }
    if constexpr (VEC) {
        if (e0 < d) *(vec_t<T, 4> *)(row + e0) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e0 + j < d) row[e0 + j] = v.e[j];
    }
}
// all elements of an owned row from the accumulators of at_columns
template <class T, bool VEC, int ND> __device__ __forceinline__ void at_store(T *row, int d, int t0, const f32x16_t (&acc)[ND], float by, int lane)
{
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            at_store4<T, VEC>(row, 32 * (t0 + t) + 8 * g + 4 * (lane >> 5), d, acc[t][4 * g] * by, acc[t][4 * g + 1] * by, acc[t][4 * g + 2] * by,
                              acc[t][4 * g + 3] * by);
}

// What rounding to bf16 takes from a float: the difference of the two as numbers of 32 bits, in units of 2^8, and back
__device__ __forceinline__ int at_low(float x)
{
    const int bits = (int)__float_as_uint(x), high = (int)(pack_bf16(x, 0.0f) << 16);
    return min((bits - high + 128) >> 8, 127);
}
__device__ __forceinline__ float at_whole(uint32_t high, int low) { return __uint_as_float((high << 16) + ((uint32_t)low << 8)); }
template <int ND> __device__ __forceinline__ void at_store_low(int8_t *row, int d, const f32x16_t (&acc)[ND], float by, int lane)
{
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = 32 * t + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
            if (e < d) row[e] = (int8_t)at_low(acc[t][i] * by);
        }
}

// The rows of a wave, through LDS, so that lanes next to each other write what is next to each other (a lane has four neighbouring elements of its
// row at a time; forward, 4 x 4096 positions, causal, 32 / 8 heads of 128, two places for the output: 674 us from the registers, 645 so).
// own: kAtOwn<DP> bytes of LDS that are this wave's alone; to: its first row, rows: how many there are; d a multiple of 8.
template <int DP> constexpr int kAtOwn = 32 * (2 * DP + 16);
template <int DP, int ND>
__device__ __forceinline__ void at_store_rows(unsigned char *own, bf16_t *to, bf16_t *to2, size_t stride, int rows, int d, const f32x16_t (&acc)[ND], float by,
                                              int lane)
{
    constexpr int CH = DP / 8, RB = 2 * DP + 16;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const chunk8 c = {pack_bf16(acc[t][4 * g] * by, acc[t][4 * g + 1] * by), pack_bf16(acc[t][4 * g + 2] * by, acc[t][4 * g + 3] * by)};
            *(chunk8 *)(own + (lane & 31) * RB + 2 * (32 * t + 8 * g + 4 * (lane >> 5))) = c;
        }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i0 = 0; i0 < 32 * CH; i0 += 64) {
        const int i = i0 + lane, row = i / CH, c = i % CH;
        if (row >= rows || 8 * c >= d) continue;
        const chunk16 v = *(const chunk16 *)(own + row * RB + 16 * c);
        *(chunk16 *)(to + row * stride + 8 * c) = v;
        if (to2) *(chunk16 *)(to2 + row * stride + 8 * c) = v;
    }
}
template <int DP, int ND>
__device__ __forceinline__ void at_store_low_rows(unsigned char *own, int8_t *to, size_t stride, int rows, int d, const f32x16_t (&acc)[ND], float by, int lane)
{
    constexpr int CH = DP / 8, RB = DP + 8;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            int low[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) low[j] = at_low(acc[t][4 * g + j] * by);
            *(uint32_t *)(own + (lane & 31) * RB + 32 * t + 8 * g + 4 * (lane >> 5)) = (low[0] & 255) | (low[1] & 255) << 8 | (low[2] & 255) << 16 | (uint32_t)low[3] << 24;
        }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i0 = 0; i0 < 32 * CH; i0 += 64) {
        const int i = i0 + lane, row = i / CH, c = i % CH;
        if (row < rows && 8 * c < d) *(chunk8 *)(to + row * stride + 8 * c) = *(const chunk8 *)(own + row * RB + 8 * c);
    }
}

// Calls F<T, DP, VEC, EXTRA, HALF> for a shape.  Heads of a width that is no multiple of 16 bytes are read element by element.
// bf16 heads take the next multiple of 32 or 64; float and element-wise ones, of which fewer kernels are built, 64, 128 or 256.
// HALF: queries and keys are 16-bit floats (AttnArgs::half).
template <template <class, int, bool, bool, bool> class F, class... A> hipError_t at_dispatch(int dt, const AttnArgs &p, const A &...a)
{
    const AttnShape &s = p.s;
    const bool extra = s.cap > 0.0f || s.bias != 0, vec = s.d % (16 / (int)dt_size(dt)) == 0;
    const int d = s.d;
#define AT_GO(T, DP, VEC, EXTRA, HALF) return F<T, DP, VEC, EXTRA, HALF>::go(p, a...)
    if (dt == DT_F32) {
        if (vec) { if (d <= 64) AT_GO(float, 64, true, true, false); if (d <= 128) AT_GO(float, 128, true, true, false); AT_GO(float, 256, true, true, false); }
        if (d <= 64) AT_GO(float, 64, false, true, false);
        if (d <= 128) AT_GO(float, 128, false, true, false);
        AT_GO(float, 256, false, true, false);
    }
#define AT_ODD(DP) if (d <= DP) { if (p.half) AT_GO(bf16_t, DP, false, true, true); AT_GO(bf16_t, DP, false, true, false); }
#define AT_BF16(DP)                                                                                                \
    if (d <= DP) {                                                                                                 \
        if (p.half) { if (extra) AT_GO(bf16_t, DP, true, true, true); AT_GO(bf16_t, DP, true, false, true); }      \
        if (extra) AT_GO(bf16_t, DP, true, true, false);                                                           \
        AT_GO(bf16_t, DP, true, false, false);                                                                     \
    }
    if (!vec) { AT_ODD(64) AT_ODD(128) AT_ODD(256) return hipErrorInvalidValue; }
    AT_BF16(32) AT_BF16(64) AT_BF16(96) AT_BF16(128) AT_BF16(192) AT_BF16(256)
#undef AT_BF16
#undef AT_ODD
#undef AT_GO
    return hipErrorInvalidValue;
}

template <class K> hipError_t at_launch(K kernel, int blocks, int smem, const AttnArgs &a, hipStream_t stream)
{
    if (smem > (48 << 10)) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(AT_TPB), smem, stream, a);
    return hipGetLastError();
}

}  // namespace bapipe
