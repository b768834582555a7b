// What the attention kernels share: matrix instructions, tiles of 16-bit rows in LDS, sequences packed one after the other.
#pragma once
#include "s24_lds.h"

#define S24_TRY(call)                           \
    do {                                        \
        const int status_ = (call);             \
        if (status_ != S24_OK) return status_;  \
    } while (0)

namespace s24_attn {
using namespace s24_lds;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

// 16 x 16 x 32: lane l holds row (A) or column (B) l%16, its elements 8*(l/16) .. + 7 of the contraction; accumulator i is row
// 4*(l/16) + i of column l%16.
template <typename T> __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma<uint16_t>(uint4 a, uint4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma<s24_half>(uint4 a, uint4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two values to 16 bits each, to nearest even.  (As conversions that the compiler knows, not as an instruction written out: between an exponential or a matrix
// instruction and what uses its result, it has to put the wait that the hardware asks for.)
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<uint16_t>(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
template <> __device__ __forceinline__ uint32_t pack2<s24_half>(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
}
// Two accumulators of neighbouring 16-row tiles as one operand of the next product: element j of lane group g is row 4g + j of the first for
// j < 4 and row 4g + j - 4 of the second otherwise, which `columns` below matches.
template <typename T> __device__ __forceinline__ uint4 operand(f32x4 a, f32x4 b)
{
    return make_uint4(pack2<T>(a[0], a[1]), pack2<T>(a[2], a[3]), pack2<T>(b[0], b[1]), pack2<T>(b[2], b[3]));
}

// What such an operand leaves of the accumulators: a second operand, which gives a product 16 bits of them.  The gradients of the queries and keys take dS so: rounded
// once it costs them as much as the rounding of their results does.  Both passes of 8192 tokens, 64 heads on 8 of 128, take 15 % longer for it.
template <typename T> __device__ __forceinline__ uint4 rest(uint4 x, f32x4 a, f32x4 b)
{
    using Num = s24_num<T>;
    // (Of binary16 as a product with -1 that the compiler does not know: an fma converts its operand itself, a subtraction does not.  2 % of the gradients' time.)
    float minus = -1.0f;
    if (!std::is_same<T, uint16_t>::value) asm("" : "+v"(minus));
    auto less = [&](float value, float held) { return std::is_same<T, uint16_t>::value ? value - held : fmaf(held, minus, value); };
    return operand<T>(f32x4{less(a[0], Num::lo(x.x)), less(a[1], Num::hi(x.x)), less(a[2], Num::lo(x.y)), less(a[3], Num::hi(x.y))},
                      f32x4{less(b[0], Num::lo(x.z)), less(b[1], Num::hi(x.z)), less(b[2], Num::lo(x.w)), less(b[3], Num::hi(x.w))});
}

// Rows of 16 lanes: the odd rows of a and the even rows of b change places / the last two of a and the first two of b
__device__ __forceinline__ void swap_rows(uint32_t &a, uint32_t &b)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto v = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = v[0], b = v[1];
#endif
}
__device__ __forceinline__ void swap_halves(uint32_t &a, uint32_t &b)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto v = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = v[0], b = v[1];
#endif
}
// x[j] of row r <-> x[r] of row j (its own inverse)
__device__ __forceinline__ void transpose_rows(uint32_t (&x)[4])
{
    swap_halves(x[0], x[2]), swap_halves(x[1], x[3]), swap_rows(x[0], x[1]), swap_rows(x[2], x[3]);
}
// Their lowest bytes
__device__ __forceinline__ uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// What a stored value left of x: the difference of their bits as fp32, in 256ths of the stored value's last place, -128 .. 127.  (Of binary16 below 2^-14, whose
// last places are further apart, what does not fit is left out.)
template <typename T> struct Left;
template <> struct Left<uint16_t> { static constexpr int kShift = 8; };
template <> struct Left<s24_half> { static constexpr int kShift = 5; };
template <typename T> __device__ __forceinline__ uint32_t left_of(float x, float stored)
{
    constexpr int S = Left<T>::kShift;
    return (uint32_t)((min(max((int)(__float_as_uint(x) - __float_as_uint(stored)), -(128 << S)), (127 << S) + (1 << (S - 1)) - 1) + (1 << (S - 1))) >> S);
}
template <typename T> __device__ __forceinline__ uint32_t four_left(f32x4 x, uint2 stored)
{
    using Num = s24_num<T>;
    return four_bytes(left_of<T>(x[0], Num::lo(stored.x)), left_of<T>(x[1], Num::hi(stored.x)), left_of<T>(x[2], Num::lo(stored.y)), left_of<T>(x[3], Num::hi(stored.y)));
}
// The other way: a stored value with what it left, of which byte i of `four` tells
template <typename T> __device__ __forceinline__ float with_left(float stored, uint32_t four, int i)
{
    return __uint_as_float(__float_as_uint(stored) + ((uint32_t)(int)(int8_t)(four >> (8 * i)) << Left<T>::kShift));
}
// Sum over eight values of x times y, of which x has the rests `left`
template <typename T> __device__ __forceinline__ float dot(uint4 x, uint2 left, uint4 y)
{
    using Num = s24_num<T>;
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t four = e < 2 ? left.x : left.y;
        sum = fmaf(with_left<T>(Num::lo(xs[e]), four, 2 * (e & 1)), Num::lo(ys[e]), fmaf(with_left<T>(Num::hi(xs[e]), four, 2 * (e & 1) + 1), Num::hi(ys[e]), sum));
    }
    return sum;
}

// A tile of rows of D 16-bit values in LDS.  It is read in two ways, neither with bank conflicts: 16-byte pieces of 16 rows, of which the LDS takes rows 0-3 and
// 12-15 of one piece together with rows 4-11 of the next in a cycle, and transposed, 8 rows at two neighbouring pieces.  Hence piece c of a row lies at slot
// c ^ (twice its place among eight).
template <int D> __device__ __forceinline__ int swizzle(int row)
{
    static_assert(D == 64 || D == 128, "rows of half a round of the banks, or of one");
    return D == 128 ? (row & 7) << 1 : (row >> 1 & 3) << 1;
}
// Byte offset in a tile of piece c of `row`
template <int D> __device__ __forceinline__ int piece(int row, int c) { return row * 2 * D + ((c ^ swizzle<D>(row)) << 4); }
// 16 rows from `row` on, elements 32*k .. + 31: an operand whose rows (columns) are the tile's rows
template <int D> __device__ __forceinline__ uint4 rows(const lds_byte *tile, int row, int k, int lane)
{
    return lds_load(tile + piece<D>(row + (lane & 15), 4 * k + (lane >> 4)));
}
// 16 columns from `16*n` on of the 32 rows from `row` on: an operand that contracts over the tile's rows, in the order of `operand` above.
// (The transposing read: in a group of 16 lanes lane i points at row i/4, columns 4*(i%4) .. + 3 and receives column i of the four rows.)
template <int D> __device__ __forceinline__ uint4 columns(const lds_byte *tile, int row, int n, int lane)
{
    const int r = row + 4 * (lane >> 4) + ((lane & 15) >> 2), col = 16 * n + 4 * (lane & 3);
    struct { v4i16 a, b; } t;
#if defined(__HIP_DEVICE_COMPILE__)
    t.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(tile + piece<D>(r, col >> 3) + 2 * (col & 7)));
    t.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(tile + piece<D>(r + 16, col >> 3) + 2 * (col & 7)));
#else
    (void)r, (void)col, (void)tile, t = {};
#endif
    return __builtin_bit_cast(uint4, t);
}

// Copies of ROWS rows into such a tile by W waves: copy i of wave w fills KB w*PER + i of it.
template <int D, int ROWS, int W> struct Copy {
    static constexpr int PER = ROWS * 2 * D / 1024 / W, RPC = 512 / D;   // copies of a wave, rows of a copy
    static_assert(PER * W * 1024 == ROWS * 2 * D, "whole copies");
    uint32_t at[PER];   // a lane's byte offsets from the tile's first row in memory
    int row0, lane, pieces, stride;
    // stride: bytes from row to row; d: the values that a row has in memory (columns past them repeat its last piece)
    __device__ __forceinline__ void init(int wave, int lane_, int stride_, int d)
    {
        row0 = wave * PER * RPC, lane = lane_, stride = stride_, pieces = d >> 3;
        offsets(ROWS);
    }
    // of a tile with `n` rows in memory, n >= 1 (rows past them repeat the last one)
    __device__ __forceinline__ void offsets(int n)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = row0 + i * RPC + lane / (D / 8), c = (lane % (D / 8)) ^ swizzle<D>(r);
            at[i] = (uint32_t)min(r, n - 1) * (uint32_t)stride + 16u * (uint32_t)min(c, pieces - 1);
        }
    }
    __device__ __forceinline__ void start(const void *first_row, lds_byte *tile) const
    {
        const rsrc_t buf = buffer_of(first_row);
#pragma unroll
        for (int i = 0; i < PER; ++i) buffer_to_lds<16>(buf, (lds_ptr)(tile + (row0 * 2 * D + i * 1024)), at[i]);
    }
};

// A sequence's part of packed tokens; whatever the offsets hold, it lies within them.
struct Span { int first, count; };
__device__ __forceinline__ Span span(const int *cu, int i, int tokens)
{
    const int a = min(max(cu[i], 0), tokens), b = min(max(cu[i + 1], a), tokens);
    return {a, b - a};
}

// Sum over this lane and those before it: within rows of 16, then from row to row, in the vector registers
__device__ __forceinline__ int running_sum(int x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // the last lane of a row to the next
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // of the first half to the second
#endif
    return x;
}
// Item t of lists that lie one after the other, `sizes(i)` long for i = 0 .. n - 1: its list, its place in it and the list's length; false past the last.
// Every wave looks for itself, 64 lists at a time.
template <typename Sizes> __device__ __forceinline__ bool find_item(int n, int t, int lane, int &list, int &place, int &length, Sizes sizes)
{
    for (int base = 0; base < n; base += 64) {
        const int size = base + lane < n ? sizes(base + lane) : 0, sum = running_sum(size);
        const unsigned long long past = __ballot(t < sum);
        if (past != 0) {
            const int owner = __ffsll(past) - 1;
            list = __builtin_amdgcn_readfirstlane(base + owner);
            length = __builtin_amdgcn_readlane(size, owner);
            place = t - (__builtin_amdgcn_readlane(sum, owner) - length);
            return true;
        }
        t -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}
// The sequence that tile t belongs to, and which of its tiles it is, where a sequence of n rows has ceil(n / rows) tiles
__device__ __forceinline__ bool find_tile(const int *cu, int sequences, int tokens, int rows, int t, int lane, int &sequence, int &index, int &count)
{
    return find_item(sequences, t, lane, sequence, index, count, [&](int i) { return (span(cu, i, tokens).count + rows - 1) / rows; });
}

// The same for tiles that take unequal time, the longest of all sequences first, so that a launch does not end with a few long ones.  A sequence's tiles are
// counted from its longest: tile j is of length min(longest, from - j), and there are `tiles`.  `at` is then j.  Found is the length L of which and above which
// there are more than t tiles, and above which there are not.  Not `mixed`, or more sequences than a wave holds lengths of: one sequence after the other.
struct Lengths { int tiles, from, longest; };
template <typename Of> __device__ __forceinline__ bool find_by_length(bool mixed, int n, int t, int most, int lane, int &list, int &at, Of of)
{
    int count;
    if (!mixed || n > 64) return find_item(n, t, lane, list, at, count, [&](int i) { return of(i).tiles; });
    const Lengths mine = lane < n ? of(lane) : Lengths{0, 0, 0};
    auto above = [&](int length) { return length < mine.longest ? min(max(mine.from - length, 0), mine.tiles) : 0; };
    auto sum = [](int x) { return __builtin_amdgcn_readlane(running_sum(x), 63); };
    if (t >= sum(above(0))) return false;
    int lo = 0, hi = most;   // more than t tiles are longer than lo, no more than t longer than hi
    while (hi - lo > 1) {
        const int middle = (lo + hi) >> 1;
        if (sum(above(middle)) > t) lo = middle;
        else hi = middle;
    }
    const int before = above(hi);
    int place;
    if (!find_item(n, t - sum(before), lane, list, place, count, [&](int) { return above(hi - 1) - before; })) return false;
    at = __builtin_amdgcn_readlane(before, list) + place;
    return true;
}

// Workgroups are dealt round-robin to the eight XCDs: head of the workgroup at place s of a row of `heads`, such that an XCD has neighbouring ones, which
// share keys and values in its L2.
__device__ __forceinline__ int head_of(int s, int heads) { return heads % 8 == 0 ? (s & 7) * (heads >> 3) + (s >> 3) : s; }

// For the scheduler: the LDS reads of a product come a step ahead of its matrix instructions, of which there are STEPS times MATRIX, READS for each.  (Left to itself
// it reads two operands, waits for them, and multiplies: the forward pass of 8192 tokens, 64 heads on 8 of 128, takes 970 us so and 950 with this.  Heads of 64
// have too few steps for it: 31.5 us with it, 30.7 without, 8 x 1024 tokens of 12 heads.  In the sums of dK and dV it takes the gradients of 9 ragged sequences of 16
// heads on 4 of 128 from 116 us to 111, in the other products of the backward pass nothing or less.)
template <int READS, int MATRIX, int STEPS> __device__ __forceinline__ void reads_ahead()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * READS, 0);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, MATRIX, 0);
        if (i + 2 < STEPS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
#endif
}

// Which tile, head and part a workgroup has
struct Unit { int tile, head, part; };
__device__ __forceinline__ Unit unit_of(unsigned block, int heads, int parts)
{
    const int units = heads * parts, tile = block / units, unit = head_of(block - tile * units, units), head = unit / parts;
    return {tile, head, unit - head * parts};
}
// The rows of a workgroup that goes over the keys of a key-value head: the queries of the head's whole group, token by token.  So a tile's rows see almost the same
// keys, and a sequence of few tokens fills a tile with those of several heads.  (512, 446 and 43 tokens after 4700 to 7400, 64 heads on 8 of 128: 309 us with one
// head to a tile, 245 so; 8192 tokens of one sequence take the same.)
struct Queries {
    Span q, k;
    int rows, row0, token0, extra, ahead;   // of the sequence; first one of the workgroup, its token, its place among the token's; token i sees the keys up to i + ahead
    int seen, wave_seen, wave_all;          // keys that some row of the workgroup may see, that one of the wave may see, that all of them see
    float inverse;
    __device__ __forceinline__ void init(Span queries, Span keys, int group, bool causal, int tile, int rows_of_tile, int first_of_wave)
    {
        q = queries, k = keys;
        rows = q.count * group, row0 = tile * rows_of_tile, token0 = row0 / group, extra = row0 - token0 * group, ahead = k.count - q.count;
        inverse = 1.0f / (float)group;
        const int w0 = row0 + first_of_wave;
        auto up_to = [&](int row) { return causal ? min(k.count, token0 + place_of(row - row0) + 1 + ahead) : k.count; };
        seen = up_to(min(row0 + rows_of_tile, rows) - 1);
        wave_seen = w0 < rows ? up_to(min(w0 + 32, rows) - 1) : 0;
        wave_all = w0 + 32 > rows ? 0 : up_to(w0);
        seen = __builtin_amdgcn_readfirstlane(seen), wave_seen = __builtin_amdgcn_readfirstlane(wave_seen), wave_all = __builtin_amdgcn_readfirstlane(wave_all);
    }
    // Tokens from the workgroup's first one to that of its row i.  (Half a step of the quotient is far more than the product's rounding: i + extra < 2^17.)
    __device__ __forceinline__ int place_of(int i) const { return (int)(((float)(i + extra) + 0.5f) * inverse); }
    // Token (of the packed ones), place in the sequence and head of the workgroup's row i; of its last one for those past the sequence
    struct Row { int64_t token; int at, head; };
    __device__ __forceinline__ Row row(int group, int kv, int i) const
    {
        const int mine = min(i, rows - 1 - row0), place = place_of(mine);
        return {q.first + token0 + place, token0 + place, kv * group + mine + extra - place * group};
    }
};

// Sum / maximum over the four lanes of a column
__device__ __forceinline__ float column_sum(float x) { x += __shfl_xor(x, 16); return x + __shfl_xor(x, 32); }
__device__ __forceinline__ float column_max(float x) { x = fmaxf(x, __shfl_xor(x, 16)); return fmaxf(x, __shfl_xor(x, 32)); }

// Scores whose maximum grew by less than this (as a power of two) keep the reference they have: P then reaches 2^8, which the 16-bit types hold with
// the same relative precision, and the sums stay far inside fp32.
constexpr float kGrowth = 8.0f;

// Rows of a join: a workgroup takes a few of a sequence, for one head
constexpr int kJoinRows = 16;
struct Joined { int64_t first; int rows, head; };
__device__ __forceinline__ bool join_rows(const int *cu, int sequences, int tokens, int heads, Joined &j)
{
    const int tile = blockIdx.x / heads;
    int sequence, index, count;
    if (!find_tile(cu, sequences, tokens, kJoinRows, tile, threadIdx.x & 63, sequence, index, count)) return false;
    const Span s = span(cu, sequence, tokens);
    j = {s.first + (int64_t)index * kJoinRows, min(kJoinRows, s.count - index * kJoinRows), (int)(blockIdx.x - tile * heads)};
    return true;
}

// ---- host
inline int check_rows(const s24_heads *v, int64_t tokens, int64_t heads, int64_t d, bool written)
{
    S24_REQUIRE(v != nullptr && (v->data != nullptr || tokens == 0), S24_ERR_NULL);
    S24_REQUIRE(v->token >= 0 && v->head >= 0 && v->token < 1 << 23 && v->head < (int64_t)1 << 46, S24_ERR_SHAPE);
    S24_REQUIRE(s24_aligned(v->data, 16) && v->token % 8 == 0 && v->head % 8 == 0, S24_ERR_ALIGN);
    if (written && tokens > 1) S24_REQUIRE(v->token >= d, S24_ERR_SHAPE);
    if (written && heads > 1) S24_REQUIRE(v->head >= d, S24_ERR_SHAPE);
    if (written && tokens > 1 && heads > 1)   // one of the two axes lies within a step of the other: no two rows share an element
        S24_REQUIRE(v->token >= (heads - 1) * v->head + d || v->head >= (tokens - 1) * v->token + d, S24_ERR_SHAPE);
    return S24_OK;
}
// Workgroups for tiles of `rows` of packed sequences: no more tiles than this, however the tokens are shared out.
inline int64_t most_tiles(int64_t tokens, int64_t sequences, int rows) { return tokens / rows + (tokens < sequences ? tokens : sequences); }
// Workgroups of 256 that a launch takes
constexpr int64_t kMostGroups = kMostItems / 256;

// How the work of a launch is cut up.  A workgroup's steps follow each other, and when causal the last queries (the first keys) take twice the average: few
// workgroups, or some with many steps, leave most of the device idle.  So what a tile sums over is cut into parts, whose sums go through memory in fp32
// for another launch to add: as many parts as make the estimate the least.  `groups` workgroups have `steps` steps of `us` microseconds each, of which `busy`
// are taken on average, and a part's sums take `bytes` bytes: the time is that of the longest, or of all of them on the device, two a compute unit, and 5 us for the
// second launch and 5 bytes a picosecond for sums that are written and read.  (On operands that are in no cache, in one part and in the best of 2, 4 and 8.
// Forward: 1 head of 64, 8192 tokens 134 us and 34 in 8; 8 heads of 128 on 2, 40 tokens after 8000: 190 and 41 in 8; 64 on 8, 512 after 3500: 111 and 92
// in 2; 32 of 128, 1500 tokens 47 and 54 in 2; the estimate takes the better one in 15 of 16 shapes.)
inline int parts_for(double groups, double steps, double busy, double us, double bytes)
{
    int best = 1;
    double least = 0.0;
    for (int p = 1; p <= 16; p *= 2) {
        const double rounds = groups * p * busy / (2.0 * s24_cu_count());
        const double t = us * steps / p * (rounds > 1.0 ? rounds : 1.0) + (p > 1 ? 5.0 + p * bytes * 2.0 / 5e6 : 0.0);
        if (p == 1 || t < least) best = p, least = t;
    }
    return best;
}

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
}  // namespace s24_attn
