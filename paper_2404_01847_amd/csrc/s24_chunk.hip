// Attention of new tokens over the paged key-value cache: the last tokens of each sequence, which the cache has, attend to all of its positions.
//
// The formulas and the structure are those of the forward pass over packed sequences (s24_attn.hip): tiles of 128 rows (the queries of a group of heads, token by
// token), four waves of 32, against tiles of 64 positions in two LDS buffers, one pass with the running maximum and sum of each row.  The positions come from their pages:
// a wave brings sixteen of a tile, which lie in one page.
// S^T = K Q^T has positions as rows, in such an order that a lane's weights are those of 16 consecutive ones: row 4g + r of the tile's t-th sixteen is position 16g + 4t + r.  V
// lies in its page with 8 (16) tokens of a channel in a piece, which is what the second product contracts along, so V needs no transposing read.
// 8 bits: whole numbers become binary16 on their way into LDS; the steps of K are factors of the scores, those of V of the weights, against a reference that has the largest
// step so far as a factor (as in the attention of one token).
#include "s24_kv.h"

#include <math.h>

namespace s24_kv {
struct ChunkArgs {
    Cache c;
    Strided q, o;
    const int *cu, *table, *lengths;
    int64_t width;
    int sequences, tokens, group, causal;
    int pieces, round; // that the tiles of a key-value head are cut into at most, 0: none is cut; as many of them as the device holds workgroups
    int sum_rows;      // that a workgroup adds the parts of
    float scale;
    float2 *weights;   // [hkv][pieces][kChunkRows]: reference and sum
    float *sums;       // [hkv][pieces][kChunkRows][d]
};
constexpr int kChunkRows = 128, kChunkKeys = 64;
__device__ __forceinline__ Span keys_of(const ChunkArgs &a, int i) { return {0, min(max(a.lengths[i], 0), (int)(a.width << a.c.shift))}; }
__device__ __forceinline__ int row_tiles(const ChunkArgs &a, int i) { return (int)(((int64_t)span(a.cu, i, a.tokens).count * a.group + kChunkRows - 1) / kChunkRows); }
__device__ __forceinline__ int key_tiles(const ChunkArgs &a, int i) { return (keys_of(a, i).count + kChunkKeys - 1) / kChunkKeys; }
// Where tiles of rows are few, the positions that they go over are cut into parts, those of a sequence of one size, which leave their sums for another kernel to add; a tile in one part
// is finished where it is.  A part has about `each` steps (tiles of positions): as few as make no more pieces than the device holds workgroups, two to a compute unit.  (12
// sequences of 2 to 512 tokens after up to 4000, 32 heads on 8 of 128, 43 tiles of 35 to 62 steps: uncut 142 us, so 112 to 115.  Steps dealt out evenly, whatever tiles they belong
// to, 157: a piece costs 5 to 10 us besides its steps.)  Where the tiles do not go evenly into them, so that the last piece would end more than a quarter later than an even share of all
// steps, and eight steps, they are cut into twice as many pieces, of which a compute unit takes the next when it is done with one (the same batch after up to 12000: 310 us in one
// round, 242 in two; with 32 heads on 2, after 8000, 184 and 153; where the pieces come out even, 512 tokens after 16000, 140 and 158).
constexpr int kFewRows = 32;      // of a sequence
// Least steps of a part, and where the longest sequence has at least so many.  (One sequence of 16000 positions, 4 heads on 1 of 128: 20.5 us with eight, 18.4 with six; 58 of up to 652, 16 heads
// on 8 of 64, are better off in one part: 20 us and 22.)
constexpr int kLeastSteps = 8, kLeastOfLong = 6, kLong = 32;
constexpr int kCutSteps = kLeastSteps + kLeastSteps / 2;   // of the shortest sequence in two parts
constexpr int kRound = 8;         // steps that a second round costs
__device__ __forceinline__ bool is_few(const ChunkArgs &a, int i) { return (int64_t)span(a.cu, i, a.tokens).count * a.group <= kFewRows; }
__device__ __forceinline__ int lanes_sum(int x) { return __builtin_amdgcn_readlane(running_sum(x), 63); }
// Largest of what the lanes have, none of it negative
__device__ __forceinline__ int lanes_max(int x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));   // the last lane of a row to the next
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));   // of the first half to the second
#endif
    return __builtin_amdgcn_readlane(x, 63);
}
struct Parts { int count, steps; };   // of a tile of a sequence, and the steps of each
__device__ __forceinline__ Parts parts_in(int keys, int each)
{
    const int count = max(1, (int)((2 * (unsigned)keys + each) / (2 * (unsigned)each)));
    return {count, (keys + count - 1) / count};
}
// The sequences as the cutting sees them.  Up to 64 of them are looked at once, a lane each.
struct Extent { int tiles, keys, few; };   // of rows, of positions
struct Cutting {
    const ChunkArgs &a;
    int lane;
    Extent mine;
    __device__ __forceinline__ Cutting(const ChunkArgs &args, int of_lane) : a(args), lane(of_lane) { mine = lane < a.sequences ? look(lane) : Extent{0, 0, 0}; }
    __device__ __forceinline__ Extent look(int i) const { return {row_tiles(a, i), key_tiles(a, i), is_few(a, i)}; }
    // That of sequence i, by the lane that has it in turn
    __device__ __forceinline__ Extent in_turn(int i) const { return a.sequences <= 64 ? mine : look(i); }
    // That of a sequence which is the same for all lanes
    __device__ __forceinline__ Extent of(int i) const
    {
        if (a.sequences > 64) return look(i);
        return {__builtin_amdgcn_readlane(mine.tiles, i), __builtin_amdgcn_readlane(mine.keys, i), __builtin_amdgcn_readlane(mine.few, i)};
    }
    // Least steps of a part that make no more than so many pieces
    __device__ __forceinline__ int least_steps(int pieces, int tiles, int all, int longest) const
    {
        const int least = longest >= kLong ? kLeastOfLong : min(kLeastSteps, longest);
        // (A tile of x times as many steps has no more than x parts besides its first: all of them at most as many as pieces are left.)
        if (a.sequences > 64) return tiles == pieces ? longest : max(all / (pieces - tiles) + 1, least);
        int lo = max(all / pieces, least), hi = max(longest, lo);   // `hi` makes few enough pieces
        while (lo < hi) {
            const int middle = (lo + hi) >> 1;
            if (lanes_sum(mine.tiles * parts_in(mine.keys, middle).count) <= pieces) hi = middle;
            else lo = middle + 1;
        }
        return hi;
    }
    // Steps of a part
    __device__ __forceinline__ int each() const
    {
        int64_t steps = 0;
        int longest = 0, tiles = 0;
        for (int i = lane; i < a.sequences; i += 64) {
            const Extent x = in_turn(i);
            steps += (int64_t)x.tiles * x.keys, tiles += x.tiles, longest = x.tiles > 0 ? max(longest, x.keys) : longest;
        }
        longest = max(lanes_max(longest), 1);
        if (longest < kCutSteps) return longest;
        tiles = lanes_sum(tiles);
        const int high = lanes_sum((int)min(steps >> 12, (int64_t)1 << 24)), low = lanes_sum((int)(steps & 4095));
        // (More steps than the host has seen to have offsets that do not ascend: then nothing is cut.)
        if (high > 1 << 18 || tiles > a.pieces) return longest;
        const int all = (high << 12) + low, once = tiles <= a.round ? least_steps(a.round, tiles, all, longest) : longest;
        if (a.pieces == a.round) return once;
        // When one round would end
        const int even = all / a.round, half = a.sequences > 64 ? min(longest, once + once / 2) : lanes_max(mine.tiles > 0 ? parts_in(mine.keys, once).steps : 0);
        const int last = tiles <= a.round ? half : even + longest / 2;
        return last > even + even / 4 + kRound ? least_steps(a.pieces, tiles, all, longest) : once;
    }
    // Sums that the sequences before this one leave
    __device__ __forceinline__ int slots_before(int each, int sequence) const
    {
        int before = 0;
        for (int i = lane; i < sequence; i += 64) {
            const Extent x = in_turn(i);
            const int count = parts_in(x.keys, each).count;
            before += count > 1 ? x.tiles * count : 0;
        }
        return lanes_sum(before);
    }
};
// A workgroup's work: steps begin .. end - 1 of a tile of rows (its steps are all of the sequence's); where its sums go, or -1: to O
struct Piece { int sequence, tile, begin, end, slot; };
// Piece t of those of a key-value head: the longest come first, and those of few rows last; of a sequence all tiles' first parts, then all tiles' next ones, so that workgroups which
// run at the same time read the same positions.
__device__ __forceinline__ bool find_part(const ChunkArgs &a, int t, int lane, Piece &piece)
{
    const Cutting cutting(a, lane);
    const int each = cutting.each(), most = (int)((a.width << a.c.shift) / kChunkKeys) + 2;
    int wide = 0, sequence, at;
    for (int i = lane; i < a.sequences; i += 64) {
        const Extent x = cutting.in_turn(i);
        wide += x.few ? 0 : x.tiles * parts_in(x.keys, each).count;
    }
    wide = lanes_sum(wide);
    const bool few = t >= wide;
    auto of = [&](int i) {
        const Extent x = cutting.in_turn(i);
        const Parts p = parts_in(x.keys, each);
        return x.few == few ? Lengths{x.tiles * p.count, INT32_MAX, max(p.steps, 1)} : Lengths{0, 0, 0};
    };
    if (!find_by_length(true, a.sequences, few ? t - wide : t, most, lane, sequence, at, of)) return false;
    const Extent x = cutting.of(sequence);
    const Parts p = parts_in(x.keys, each);
    const int part = at / max(x.tiles, 1), slot = p.count == 1 ? -1 : cutting.slots_before(each, sequence) + at;
    piece = {sequence, x.tiles - 1 - (at - part * x.tiles), part * p.steps, min(x.keys, (part + 1) * p.steps), slot};
    return at >= 0 && part < p.count && slot < a.pieces;   // (as they are, where the offsets ascend)
}
// The workgroup's tile where each has one: a sequence, and which of its tiles, the last ones first.  The longest come first.
__device__ __forceinline__ bool find_chunk(const ChunkArgs &a, int t, int lane, Piece &piece)
{
    int sequence, at;
    auto of = [&](int i) {
        const int n = row_tiles(a, i), keys = (int)(((int64_t)keys_of(a, i).count * a.group + kChunkRows - 1) / kChunkRows);
        return a.causal ? Lengths{n, max(keys, n), INT32_MAX} : Lengths{n, INT32_MAX, max(keys, 1)};
    };
    const int64_t most = max((int64_t)a.tokens, a.width << a.c.shift) * a.group / kChunkRows + 1;
    if (!find_by_length(true, a.sequences, t, (int)most, lane, sequence, at, of)) return false;
    piece = {sequence, row_tiles(a, sequence) - 1 - at, 0, key_tiles(a, sequence), -1};
    return true;
}

// Keys of a tile in LDS: piece c of a row at slot c ^ flip.  The 16 rows of an operand are four of each sixteen positions, of which the LDS takes those of lanes 0-3 and 12-15
// of one piece together with those of lanes 4-11 of the next in a cycle.  In 8 bits rows are written every second piece at a time: there rows 4 and 5 have theirs where 0 and 1 have none.
template <int D, int BITS> __device__ __forceinline__ int flip(int row)
{
    return (D == 128 ? ((row & 3) | (row >> 4 & 1) << 2) << 1 : ((row >> 1 & 1) | (row >> 4 & 1) << 1) << 1) | (BITS == 8 ? row >> 2 & 1 : 0);
}

// A wave's sixteen positions of a tile on their way into LDS.  K [64][D], V [8][D][8]
template <int D, int BITS> struct Sixteen;
template <int D> struct Sixteen<D, 16> {
    static constexpr int PER = D / 32;   // copies of 1 KB
    uint32_t k[PER], v[PER];             // a lane's byte offsets in its page's part
    int wave;
    __device__ __forceinline__ void init(const Cache &c, int wave_, int lane)
    {
        wave = wave_;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int row = i * (512 / D) + lane / (D / 8), piece = (lane % (D / 8)) ^ flip<D, 16>(16 * wave + row);
            k[i] = (uint32_t)(row * 2 * c.d + 16 * min(piece, (c.d >> 3) - 1));
            const int at = 64 * i + lane, eight = at / D, channel = at % D;
            v[i] = (uint32_t)((eight * c.d + min(channel, c.d - 1)) * 16);
        }
    }
    // `first`: of the sixteen positions, in tokens of one head
    __device__ __forceinline__ void start(const Cache &c, int64_t first, lds_byte *tk, lds_byte *tv, float *)
    {
        const rsrc_t bk = buffer_of(c.k + first * 2 * c.d), bv = buffer_of(c.v + first * 2 * c.d);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            buffer_to_lds<16>(bk, (lds_ptr)(tk + (wave * PER + i) * 1024), k[i]);
            buffer_to_lds<16>(bv, (lds_ptr)(tv + (wave * PER + i) * 1024), v[i]);
        }
    }
    __device__ __forceinline__ void finish(lds_byte *, lds_byte *, float *, int) {}
};
template <int D> struct Sixteen<D, 8> {
    static constexpr int PER = D / 64;
    uint4 k[PER], v[PER];
    float step;
    uint32_t from_k[PER], from_v[PER];
    int wave, lane;
    // The row whose piece of 16 bytes is the at-th of the sixteen rows': 0 4 1 5 2 6 3 7 8 12 ...
    static __device__ __forceinline__ int key_row(int at) { const int i = at / (D / 16); return (i & 8) | (i & 1) << 2 | (i >> 1 & 3); }
    __device__ __forceinline__ void init(const Cache &c, int wave_, int lane_)
    {
        wave = wave_, lane = lane_;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = 64 * i + lane;
            from_k[i] = (uint32_t)(key_row(at) * c.d + 16 * min(at % (D / 16), (c.d >> 4) - 1));
            from_v[i] = (uint32_t)(min(at, c.d - 1) * 16);
        }
    }
    __device__ __forceinline__ void start(const Cache &c, int64_t first, lds_byte *, lds_byte *, float *)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            k[i] = *reinterpret_cast<const uint4 *>(c.k + first * c.d + from_k[i]);
            v[i] = *reinterpret_cast<const uint4 *>(c.v + first * c.d + from_v[i]);
        }
        step = (lane & 16 ? c.vs : c.ks)[first + (lane & 15)];
    }
    // `left`: how many of the positions the sequence has.  (What lies past its end may hold anything: there V has the step 0.)
    __device__ __forceinline__ void finish(lds_byte *tk, lds_byte *tv, float *steps, int left)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = 64 * i + lane, row = 16 * wave + key_row(at), piece = 2 * (at % (D / 16));
            lds_byte *const to = tk + row * 2 * D;
            lds_store(to + ((piece ^ flip<D, 8>(row)) << 4), halves(k[i].x, k[i].y));
            lds_store(to + (((piece + 1) ^ flip<D, 8>(row)) << 4), halves(k[i].z, k[i].w));
            lds_store(tv + (2 * wave * D + at) * 16, halves(v[i].x, v[i].y));
            lds_store(tv + ((2 * wave + 1) * D + at) * 16, halves(v[i].z, v[i].w));
        }
        if (lane < 32) steps[(lane >> 4) * kChunkKeys + 16 * wave + (lane & 15)] = lane < 16 || (lane & 15) < left ? step : 0.0f;
    }
};

// Where a row's sums lie
__device__ __forceinline__ int64_t slot_row(const ChunkArgs &a, int kv, int slot, int row) { return ((int64_t)kv * a.pieces + slot) * kChunkRows + row; }
// The result of a row (a lane has 4 of each 16 values; `sum` of its weights): to O, or as sums
template <typename T, int E> __device__ __forceinline__ void write_row(const ChunkArgs &a, const Queries::Row &of, f32x4 (&o)[E / 16], float m, float sum, int kv, int slot, int row, bool live, int g)
{
    const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (slot < 0) {
        uint16_t *out = a.o.p + of.token * a.o.token + of.head * a.o.head;
#pragma unroll
        for (int n = 0; n < E / 16; n += 4) {   // of four such pieces of a row a lane gets one whole: lines are written with few stores
            uint32_t x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 v = n + i < E / 16 ? o[n + i < E / 16 ? n + i : 0] * inverse : f32x4{};
                x[i] = pack2<T>(v[0], v[1]), y[i] = pack2<T>(v[2], v[3]);
            }
            transpose_rows(x), transpose_rows(y);
            const int at = 16 * (n + g);
            if (at >= a.c.d || !live) continue;
            *reinterpret_cast<uint4 *>(out + at) = make_uint4(x[0], y[0], x[1], y[1]);
            *reinterpret_cast<uint4 *>(out + at + 8) = make_uint4(x[2], y[2], x[3], y[3]);
        }
    } else if (live) {
        const int64_t at = slot_row(a, kv, slot, row);
#pragma unroll
        for (int n = 0; n < E / 16; ++n)
            if (16 * n < a.c.d) *reinterpret_cast<f32x4 *>(a.sums + at * a.c.d + 16 * n + 4 * g) = o[n];
        if (g == 0) a.weights[at] = make_float2(m, sum);
    }
}

// What the reference and the sums of a row (a column of the products) are taken to when its scores grow.  In an 8-bit cache the reference has a factor for the steps of V, which
// are at most `wide`.
template <int BITS> struct Reference {
    float rise = BITS == 8 ? -100.0f : 0.0f, wide = 0x1p-100f;
    // Whether scores up to `top` (or steps up to `step`) ask for another one
    __device__ __forceinline__ bool low(float m, float top, float step) const { return top > m - rise + kGrowth || (BITS == 8 && step > wide); }
    // Its new part from the steps
    __device__ __forceinline__ float lift(float step)
    {
        if (BITS != 8) return 0.0f;
        step = column_max(step);
        if (step > wide) wide = 2.0f * step;
        return __builtin_amdgcn_logf(wide);
    }
};

// Queries as operands, and the factor of their scores.  8 bits: scaled by a power of two into what binary16 holds
template <typename T, int N> __device__ __forceinline__ float scaled_queries(uint4 (&q)[N], float c)
{
    using Num = s24_num<T>;
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k)
        for (const uint32_t x : {q[k].x, q[k].y, q[k].z, q[k].w}) most = fmaxf(most, fmaxf(fabsf(Num::lo(x)), fabsf(Num::hi(x))));
    most = column_max(most);
    const int e = most > 0.0f ? ilogbf(most) : 0;
    auto scaled = [&](uint32_t x) { return pack2<s24_half>(ldexpf(Num::lo(x), -e), ldexpf(Num::hi(x), -e)); };
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = make_uint4(scaled(q[k].x), scaled(q[k].y), scaled(q[k].z), scaled(q[k].w));
    return ldexpf(c, e);
}

// A sequence of up to 32 rows (a few tokens, such as drafted ones): each of the four waves has all of the rows and a quarter of the piece's positions, and goes over them 32 at a
// time from memory to registers, as in the attention of one token; their sums are added in LDS.  Bound by memory: 24 sequences of 6 tokens after up to 8192, 32 heads on 8 of 128, take
// 98 us, 5.9 TB/s (through LDS, as above, 131).  Kept in registers they must not spill, hence kernels for each size of a head.
// Row 4g + r of tile t of a product is position 8g + 4t + r, so that a lane's weights are those of 8 consecutive ones.
// (HEAD: values of a head, with which the addresses within a page are constants.)
template <typename T, int HEAD, int BITS, int TILE>
__device__ __forceinline__ void few_rows(const ChunkArgs &a, const Queries &s_, const int *table, int kv, int begin, int tiles, int slot, int lane, int wave, lds_byte *lds_k, lds_byte *lds_v)
{
    using M = typename std::conditional<BITS == 8, s24_half, T>::type;
    constexpr int BK = 32, d = HEAD, token = d * (BITS / 8);   // bytes of a token of one head
    constexpr int KL = BITS == 8 ? (d + 63) / 64 : (d + 31) / 32, QL = BITS == 8 ? 2 * KL : KL;
    const int col = lane & 15, g = lane >> 4;
    const int length = s_.k.count, all_units = max(min(2 * tiles, (s_.seen + BK - 1) / BK) - 2 * begin, 0);
    const int first = 2 * begin + all_units * wave / 4, end = 2 * begin + all_units * (wave + 1) / 4;

    // A unit's positions 8*(col/4) .. for K, 8*g .. for V: each sixteen lie in one page.
    auto position = [&](int t, int eight) { return min(t * BK + 16 * (eight >> 1), (length - 1) & ~15); };
    struct Pages { uint32_t k, v; };
    auto pages = [&](int t) { return Pages{(uint32_t)table[position(t, col >> 2) >> a.c.shift], (uint32_t)table[position(t, g) >> a.c.shift]}; };
    // of the sixteen, in tokens of one head
    auto place = [&](int t, int eight, uint32_t id) {
        return (((int64_t)min(id, (uint32_t)a.c.pages - 1) * a.c.hkv + kv) << a.c.shift) + (position(t, eight) & (a.c.page - 1));
    };
    typedef typename std::conditional<BITS == 8, uint2, uint4>::type Values;   // 8 positions of a channel
    typedef typename std::conditional<BITS == 8, unsigned int __attribute__((ext_vector_type(2))), s24_u32x4>::type Loaded;
    uint4 fk[2][KL];
    Values fv[d / 16];
    f32x4 sk[2], sv[2];
    auto load_k = [&](int t, Pages p) {
        const unsigned char *from = a.c.k + (place(t, col >> 2, p.k) + 8 * (col >> 2 & 1) + (col & 3)) * token;
        const float *step = a.c.ks + place(t, g, p.v) + 8 * (g & 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 0; k < KL; ++k)   // (past the head's end the query has zeros)
                fk[i][k] = s24_load_stream(from + 4 * i * token + 16 * (64 * k + 64 <= token ? 4 * k + g : min(4 * k + g, (token >> 4) - 1)));
            if (BITS == 8) sk[i] = *reinterpret_cast<const f32x4 *>(step + 4 * i);
        }
    };
    auto load_v = [&](int t, Pages p) {
        const int64_t at = place(t, g, p.v);
        const unsigned char *from = a.c.v + at * token + (BITS == 8 ? 8 * (g & 1) : (g & 1) * d * 16);
        const float *step = a.c.vs + at + 8 * (g & 1);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (BITS == 8) sv[i] = *reinterpret_cast<const f32x4 *>(step + 4 * i);
#pragma unroll
        for (int n = 0; n < d / 16; ++n) fv[n] = __builtin_bit_cast(Values, __builtin_nontemporal_load(reinterpret_cast<const Loaded *>(from + (16 * n + col) * 16)));
    };
    Pages now{}, next{};
    if (first < end) now = pages(first);
    if (first + 1 < end) next = pages(first + 1);
    uint4 q[2][QL];
    int last[2];
    float c[2];
    Queries::Row of[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        of[j] = s_.row(a.group, kv, 16 * j + col);
        last[j] = a.causal ? min(length - 1, of[j].at + s_.ahead) : length - 1;
        const uint16_t *row = a.q.p + of[j].token * a.q.token + of[j].head * a.q.head;
        c[j] = a.scale * kLog2e;
#pragma unroll
        for (int k = 0; k < QL; ++k) {
            const int i = BITS == 8 ? 64 * (k >> 1) + 16 * g + 8 * (k & 1) : 32 * k + 8 * g;
            q[j][k] = i < d ? *reinterpret_cast<const uint4 *>(row + i) : make_uint4(0, 0, 0, 0);
        }
    }
    const int all = __builtin_amdgcn_readfirstlane(last[0]) + 1;   // positions that all of the rows see: what the first one does
    if (first < end) load_k(first, now), load_v(first, now);
    if (BITS == 8) c[0] = scaled_queries<T>(q[0], c[0]), c[1] = scaled_queries<T>(q[1], c[1]);
    float m[2] = {-1e30f, -1e30f}, l[2] = {0.0f, 0.0f};
    Reference<BITS> reference;
    f32x4 o[2][d / 16];
#pragma unroll
    for (int n = 0; n < d / 16; ++n) o[0][n] = o[1][n] = f32x4{};
    // The loads run ahead: a unit's keys are asked for as soon as the scores before them are formed, its values as soon as the ones before are summed, its pages a unit before that.
    for (int t = first; t < end; ++t) {
        const Pages coming = next;
        if (t + 2 < end) next = pages(t + 2);
        const int k0 = t * BK;
        f32x4 s[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i][0] = s[i][1] = f32x4{};
#pragma unroll
            for (int k = 0; k < KL; ++k)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if constexpr (BITS == 8) {
                        s[i][j] = mma<M>(halves(fk[i][k].x, fk[i][k].y), q[j][2 * k], s[i][j]);
                        s[i][j] = mma<M>(halves(fk[i][k].z, fk[i][k].w), q[j][2 * k + 1], s[i][j]);
                    } else
                        s[i][j] = mma<M>(fk[i][k], q[j][k], s[i][j]);
                }
            if (BITS == 8) s[i][0] *= sk[i], s[i][1] *= sk[i];
        }
        if (t + 1 < end) load_k(t + 1, coming);
        if (k0 + BK > all) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[i][j][r] = k0 + 8 * g + 4 * i + r <= last[j] ? s[i][j][r] : -INFINITY;
        }
        if (k0 + BK > length) {   // what lies past the sequence's end may hold anything
            if constexpr (BITS == 8) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sv[i][r] = k0 + 8 * g + 4 * i + r < length ? sv[i][r] : 0.0f;
            } else {
#pragma unroll
                for (int n = 0; n < d / 16; ++n) {
                    uint32_t *x = reinterpret_cast<uint32_t *>(&fv[n]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int left = length - (k0 + 8 * g + 2 * i);
                        x[i] = left >= 2 ? x[i] : left == 1 ? x[i] & 0xFFFFu : 0u;
                    }
                }
            }
        }
        float top[2], step = 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            top[j] = s[0][j][0];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) top[j] = fmaxf(top[j], s[i][j][r]);
            top[j] *= c[j];
        }
        if (BITS == 8) step = fmaxf(fmaxf(fmaxf(sv[0][0], sv[0][1]), fmaxf(sv[0][2], sv[0][3])), fmaxf(fmaxf(sv[1][0], sv[1][1]), fmaxf(sv[1][2], sv[1][3])));
        if (__any(reference.low(m[0], top[0], step) || reference.low(m[1], top[1], step))) {
            const float before = reference.rise, lift = reference.lift(step);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float now = fmaxf(m[j] - before, column_max(top[j])) + lift, shrink = __builtin_amdgcn_exp2f(m[j] - now);
                m[j] = now, l[j] *= shrink;
#pragma unroll
                for (int n = 0; n < d / 16; ++n) o[j][n] *= shrink;
            }
            reference.rise = lift;
        }
        uint4 p[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c[j], -m[j]));
                    l[j] += s[i][j][r];
                }
                if (BITS == 8) s[i][j] *= sv[i];
            }
            p[j] = operand<M>(s[0][j], s[1][j]);   // rounded to the operands' 16 bits, as the packed forward pass has it: 2^-8 (2^-11) of a weight
        }
#pragma unroll
        for (int n = 0; n < d / 16; ++n) {
            uint4 f;
            if constexpr (BITS == 8) f = halves(fv[n].x, fv[n].y);
            else f = fv[n];
            o[0][n] = mma<M>(f, p[0], o[0][n]);
            o[1][n] = mma<M>(f, p[1], o[1][n]);
        }
        if (t + 1 < end) load_v(t + 1, coming);
    }
    // The waves' sums, in order
    typedef __attribute__((address_space(3))) f32x2 lds_f32x2;
    static_assert(d / 16 * 2048 <= TILE && 3 * 1024 <= TILE, "the sums must fit");
    auto sums = [&](int w) { return w == 3 ? lds_v : lds_k + (w - 1) * TILE; };
    lds_byte *const weights = lds_v + TILE;
#pragma unroll
    for (int j = 0; j < 2; ++j) l[j] = column_sum(l[j]);
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int n = 0; n < d / 16; ++n) lds_store(sums(wave) + (j * (d / 16) + n) * 1024 + 16 * lane, o[j][n]);
            *(lds_f32x2 *)(weights + ((2 * wave - 2 + j) * 64 + lane) * 8) = f32x2{m[j], l[j]};
        }
    }
    wait_and_barrier<0>();
    if (wave > 0) return;
    for (int w = 1; w < 4; ++w)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x2 theirs = *(const lds_f32x2 *)(weights + ((2 * w - 2 + j) * 64 + lane) * 8);
            const float now = fmaxf(m[j], theirs[0]), f = __builtin_amdgcn_exp2f(m[j] - now), h = __builtin_amdgcn_exp2f(theirs[0] - now);
            m[j] = now, l[j] = fmaf(l[j], f, theirs[1] * h);
#pragma unroll
            for (int n = 0; n < d / 16; ++n) o[j][n] = o[j][n] * f + __builtin_bit_cast(f32x4, lds_load(sums(w) + (j * (d / 16) + n) * 1024 + 16 * lane)) * h;
        }
#pragma unroll
    for (int j = 0; j < 2; ++j) write_row<T, d>(a, of[j], o[j], m[j], l[j], kv, slot, 16 * j + col, 16 * j + col < s_.rows, g);
}

template <int D, int BITS> struct ChunkLds {
    static constexpr int TILE = kChunkKeys * 2 * D;
    unsigned char (&k)[2][TILE], (&v)[2][TILE];
    float (&steps)[2][BITS == 8 ? 2 * kChunkKeys : 4];
};
// D: values of a tile's row; E: values that the products go over
// HEAD: values of a head, where sequences of few rows are taken apart; 0: they are not
template <typename T, int D, int E, int BITS, int HEAD> __device__ __forceinline__ void chunk_piece(const ChunkArgs &a, const Piece &piece, int kv, int lane, int wave, const ChunkLds<D, BITS> &lds)
{
    using M = typename std::conditional<BITS == 8, s24_half, T>::type;
    constexpr int BK = kChunkKeys;
    const int col = lane & 15, g = lane >> 4;
    auto &lds_k = lds.k, &lds_v = lds.v;
    auto &steps = lds.steps;
    Queries s_;
    s_.init(span(a.cu, piece.sequence, a.tokens), keys_of(a, piece.sequence), a.group, a.causal, piece.tile, kChunkRows, 32 * wave);
    const int length = s_.k.count, all_tiles = s_.seen > 0 ? (s_.seen + BK - 1) / BK : 0, begin = piece.begin, tiles = min(all_tiles, piece.end);
    const int *table = a.table + piece.sequence * a.width;
    if constexpr (HEAD > 0) {
        if (s_.rows <= kFewRows) {
            few_rows<T, HEAD, BITS, ChunkLds<D, BITS>::TILE>(a, s_, table, kv, begin, tiles, piece.slot, lane, wave, (lds_byte *)lds_k, (lds_byte *)lds_v);
            return;
        }
    }

    // Where the wave's positions of tile t are, in tokens of one head.  (Those past the sequence's end are its last ones again.)
    auto page_of = [&](int t) {
        const int pos = min(t * BK + 16 * wave, (length - 1) & ~15);
        return min((uint32_t)table[pos >> a.c.shift], (uint32_t)a.c.pages - 1);
    };
    auto place = [&](int t, uint32_t id) {
        const int pos = min(t * BK + 16 * wave, (length - 1) & ~15);
        return (((int64_t)id * a.c.hkv + kv) << a.c.shift) + (pos & (a.c.page - 1));
    };
    uint32_t id = begin < tiles ? page_of(begin) : 0;   // of the next tile
    uint4 q[2][E / 32];
    int last[2];     // that a row sees
    float c[2];      // factor of the scores
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const Queries::Row of = s_.row(a.group, kv, 32 * wave + 16 * j + col);
        const uint16_t *row = a.q.p + of.token * a.q.token + of.head * a.q.head;
        last[j] = a.causal ? min(length - 1, of.at + s_.ahead) : length - 1;
        c[j] = a.scale * kLog2e;
#pragma unroll
        for (int k = 0; k < E / 32; ++k)
            q[j][k] = 32 * k + 8 * g < a.c.d ? *reinterpret_cast<const uint4 *>(row + 32 * k + 8 * g) : make_uint4(0, 0, 0, 0);
        if (BITS == 8) c[j] = scaled_queries<T>(q[j], c[j]);
    }
    float m[2] = {-1e30f, -1e30f}, l[2] = {0.0f, 0.0f};
    Reference<BITS> reference;
    f32x4 o[2][E / 16];
#pragma unroll
    for (int n = 0; n < E / 16; ++n) o[0][n] = o[1][n] = f32x4{};

    Sixteen<D, BITS> sixteen;
    sixteen.init(a.c, wave, lane);
    if (begin < tiles) {
        sixteen.start(a.c, place(begin, id), (lds_byte *)lds_k[begin & 1], (lds_byte *)lds_v[begin & 1], steps[begin & 1]);
        if (begin + 1 < tiles) id = page_of(begin + 1);
        sixteen.finish((lds_byte *)lds_k[begin & 1], (lds_byte *)lds_v[begin & 1], steps[begin & 1], length - begin * BK - 16 * wave);
    }
    for (int t = begin; t < tiles; ++t) {
        wait_and_barrier<0>();
        const int other = (t + 1) & 1;
        if (t + 1 < tiles) {
            sixteen.start(a.c, place(t + 1, id), (lds_byte *)lds_k[other], (lds_byte *)lds_v[other], steps[other]);
            if (t + 2 < tiles) id = page_of(t + 2);
        }
        const int k0 = t * BK;
        if (BITS == 16 && k0 + BK > length) {   // what lies past the sequence's end may hold anything: V has zeros there
            for (int i = threadIdx.x; i < 8 * D; i += 256) {
                const int left = length - k0 - 8 * (i / D);
                if (left >= 8) continue;
                lds_byte *const at = (lds_byte *)lds_v[t & 1] + 16 * i;
                uint4 x = lds_load(at);
                uint32_t *const two = reinterpret_cast<uint32_t *>(&x);
#pragma unroll
                for (int e = 0; e < 4; ++e) two[e] = left - 2 * e >= 2 ? two[e] : left - 2 * e == 1 ? two[e] & 0xFFFFu : 0u;
                lds_store(at, x);
            }
            wait_and_barrier<0>();
        }
        if (k0 < s_.wave_seen) {
            const lds_byte *tk = (const lds_byte *)lds_k[t & 1], *tv = (const lds_byte *)lds_v[t & 1];
            f32x4 s[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = f32x4{};
#pragma unroll
            for (int k = 0; k < E / 32; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * (col >> 2) + 4 * i + (col & 3);
                    const uint4 f = lds_load(tk + row * 2 * D + (((4 * k + g) ^ flip<D, BITS>(row)) << 4));
                    s[i][0] = mma<M>(f, q[0][k], s[i][0]);
                    s[i][1] = mma<M>(f, q[1][k], s[i][1]);
                }
            if (D == 128) reads_ahead<4, 8, E / 32>();
            f32x4 sv[4];
            float step = 0.0f;
            if constexpr (BITS == 8) {
                const float *now = steps[t & 1];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 sk = *reinterpret_cast<const f32x4 *>(now + 16 * g + 4 * i);
                    sv[i] = *reinterpret_cast<const f32x4 *>(now + BK + 16 * g + 4 * i);
                    s[i][0] *= sk, s[i][1] *= sk;
                    step = fmaxf(step, fmaxf(fmaxf(sv[i][0], sv[i][1]), fmaxf(sv[i][2], sv[i][3])));
                }
            }
            if (k0 + BK > s_.wave_all) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[i][j][r] = k0 + 16 * g + 4 * i + r <= last[j] ? s[i][j][r] : -INFINITY;
            }
            float top[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[j] = s[0][j][0];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top[j] = fmaxf(top[j], s[i][j][r]);
                top[j] *= c[j];
            }
            if (__any(reference.low(m[0], top[0], step) || reference.low(m[1], top[1], step))) {
                const float before = reference.rise, lift = reference.lift(step);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float now = fmaxf(m[j] - before, column_max(top[j])) + lift, shrink = __builtin_amdgcn_exp2f(m[j] - now);
                    m[j] = now, l[j] *= shrink;
#pragma unroll
                    for (int n = 0; n < E / 16; ++n) o[j][n] *= shrink;
                }
                reference.rise = lift;
            }
            uint4 p[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c[j], -m[j]));
                        l[j] += s[i][j][r];
                    }
                    if (BITS == 8) s[i][j] *= sv[i];
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) p[u][j] = operand<M>(s[2 * u][j], s[2 * u + 1][j]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < E / 16; ++n) {
                    const uint4 f = lds_load(tv + ((2 * g + u) * D + 16 * n + col) * 16);
                    o[0][n] = mma<M>(f, p[u][0], o[0][n]);
                    o[1][n] = mma<M>(f, p[u][1], o[1][n]);
                }
        }
        if (t + 1 < tiles) sixteen.finish((lds_byte *)lds_k[other], (lds_byte *)lds_v[other], steps[other], length - (t + 1) * BK - 16 * wave);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = 32 * wave + 16 * j + col;
        write_row<T, E>(a, s_.row(a.group, kv, row), o[j], m[j], column_sum(l[j]), kv, piece.slot, row, s_.row0 + row < s_.rows, g);
    }
}

// What bounds it: for many rows matrix instructions and the vector instructions of the softmax, in turn more than at once: 2 x 4096 tokens of 32 heads of 128 285 to 297 us (0.95 PFLOP/s of
// what they need, 45 and 47 % of the cycles), the same as the forward pass over packed rows takes; in 8 bits 4 chunks of 400 to 1024 tokens after up to 30000, 64 heads on 8, 2680 to 2760
// (0.9; 37 and 60 %: the whole numbers become operands once for each tile of rows).  To look for the largest score only where weights have grown past the reference saved
// instructions and lost time.
template <typename T, int D, int E, int BITS, int HEAD>
__global__ __launch_bounds__(256, 2) void chunk_kernel(const ChunkArgs a)
{
    using Lds = ChunkLds<D, BITS>;
    __shared__ __align__(16) unsigned char lds_k[2][Lds::TILE], lds_v[2][Lds::TILE];
    __shared__ __align__(16) float steps[2][BITS == 8 ? 2 * kChunkKeys : 4];
    const Lds lds{lds_k, lds_v, steps};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const Unit unit = unit_of(blockIdx.x, a.c.hkv, 1);
    Piece piece;
    if (HEAD == 0 ? !find_chunk(a, unit.tile, lane, piece) : !find_part(a, unit.tile, lane, piece)) return;
    chunk_piece<T, D, E, BITS, HEAD>(a, piece, unit.head, lane, wave, lds);
}

// O of rows whose tiles lie in several parts, from the sums that these left (those of a part past the causal diagonal have no weight).  A workgroup has a.sum_rows rows of a tile, eight
// at a time by 32 lanes each, which add four values; where it has fewer the lanes that are left take every second, fourth or eighth part.
// Bound by its chain of reads (offsets, lengths, parts): 6 us for 144 tokens of 32 heads in two or three parts, 12 for 1300.  (A workgroup for each row, which reads part after part: 40 tokens after
// 8000 81 us with the attention, 31 so.)
template <typename T>
__global__ __launch_bounds__(256) void chunk_join_kernel(const ChunkArgs a)
{
    constexpr int AT_ONCE = 4;
    __shared__ float shared[256][7];
    const int block = blockIdx.x / a.c.hkv, kv = blockIdx.x - block * a.c.hkv, lane = threadIdx.x & 63;
    int sequence, index, unused;
    if (!find_item(a.sequences, block, lane, sequence, index, unused, [&](int i) { return (int)(((int64_t)span(a.cu, i, a.tokens).count * a.group + a.sum_rows - 1) / a.sum_rows); })) return;
    const Cutting cutting(a, lane);
    const int each = cutting.each(), n = cutting.of(sequence).tiles, parts = parts_in(cutting.of(sequence).keys, each).count;
    if (parts == 1) return;
    const int before = cutting.slots_before(each, sequence);
    if (before + n * parts > a.pieces) return;
    const Span s = span(a.cu, sequence, a.tokens);
    const int row0 = index * a.sum_rows, rows = min(a.sum_rows, s.count * a.group - row0), tile = row0 / kChunkRows, d = a.c.d;
    const int64_t first = slot_row(a, kv, before + n - 1 - tile, row0 - tile * kChunkRows), step = (int64_t)n * kChunkRows;   // from part to part
    const int at_a_time = min(a.sum_rows, 8), groups = 8 / at_a_time, group = threadIdx.x / (32 * at_a_time), quad = threadIdx.x & 31, i = min(4 * quad, d - 4);
    for (int base = 0; base < rows; base += at_a_time) {
        const int row = base + (threadIdx.x >> 5) % at_a_time, of = min(row, rows - 1);
        float m = -1e30f, l = 0.0f;
        f32x4 x = {};
        for (int p = group; p < parts; p += AT_ONCE * groups) {
            float2 w[AT_ONCE];
            f32x4 v[AT_ONCE];
            float now = m;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int64_t at = first + of + min(p + u * groups, parts - 1) * step;
                w[u] = a.weights[at], v[u] = *reinterpret_cast<const f32x4 *>(a.sums + at * d + i);
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (p + u * groups >= parts) w[u].y = 0.0f;
                now = w[u].y != 0.0f ? fmaxf(now, w[u].x) : now;
            }
            const float f = __builtin_amdgcn_exp2f(m - now);
            m = now, l *= f, x *= f;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const float h = w[u].y != 0.0f ? __builtin_amdgcn_exp2f(w[u].x - now) : 0.0f;
                l = fmaf(w[u].y, h, l), x += w[u].y != 0.0f ? v[u] * h : f32x4{};
            }
        }
        if (groups > 1) {   // (then there is one turn)
            float *const mine = shared[threadIdx.x];
            mine[0] = m, mine[1] = l, mine[2] = x[0], mine[3] = x[1], mine[4] = x[2], mine[5] = x[3];
            __syncthreads();
            if (group > 0) return;
            for (int k = 1; k < groups; ++k) {
                const float *const theirs = shared[threadIdx.x + 32 * at_a_time * k];
                const float now = fmaxf(m, theirs[0]), f = __builtin_amdgcn_exp2f(m - now), h = __builtin_amdgcn_exp2f(theirs[0] - now);
                m = now, l = fmaf(l, f, theirs[1] * h), x = x * f + f32x4{theirs[2], theirs[3], theirs[4], theirs[5]} * h;
            }
        }
        if (row >= rows || 4 * quad >= d) continue;
        x *= l == 0.0f ? 0.0f : 1.0f / l;
        const int token = (row0 + row) / a.group, head = kv * a.group + row0 + row - token * a.group;
        *reinterpret_cast<uint2 *>(a.o.p + (s.first + token) * a.o.token + head * a.o.head + 4 * quad) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    }
}

// ------------------------------------------------------------------ host
// Tiles of rows of a key-value head at most, and pieces that they are cut into; 0: none is, where the sequences are short, or the rows make four whole tiles for each compute unit.  Those keep the device
// full to the end if the sequences are of like length; one that is much longer than the others then goes on alone, a workgroup for each of its tiles.  (64 heads on 8 of 128: a prompt of 1800 tokens
// beside one token after 128000 takes 313 us, of 2048 4100, the two by themselves 91 and 93; after 30000 135 and 792.  700 sequences of 6 tokens after 1000, 32 heads on 8, lose nothing: 0.77 us for
// each in whole tiles, 0.86 of 682 by the way for few rows.)
static int64_t chunk_tiles(const s24_kv_cache *c, int64_t tokens, int64_t sequences, int64_t hq)
{
    return tokens * (hq / c->hkv) / kChunkRows + (tokens < sequences ? tokens : sequences);
}
static int64_t chunk_pieces(const s24_kv_cache *c, int64_t width, int64_t tokens, int64_t sequences, int64_t hq)
{
    const int64_t held = 2 * (int64_t)s24_cu_count(), steps = (width * c->page + kChunkKeys - 1) / kChunkKeys, tiles = chunk_tiles(c, tokens, sequences, hq), rows = tokens * (hq / c->hkv);
    if (rows / kChunkRows * c->hkv >= 2 * held || tiles * steps > INT32_MAX / 2) return 0;   // (steps are counted in an int)
    // None is cut: the kernel that has a way for few rows, if most have few and more than two tiles of positions.  (16 sequences of 5 tokens after up to 500, 8 heads on 2 of 128 in 8 bits, 14 us
    // so and 20 in whole tiles; 55 of 2 tokens after none, 12 heads, 15 and 13.)
    if (steps < kCutSteps) return steps > 2 && rows <= kFewRows * sequences ? tiles : 0;
    const int64_t of_head = 2 * (held / c->hkv), worth = tiles * (1 + steps / (steps >= kLong ? kLeastOfLong : kLeastSteps));   // no more than have so many steps each
    return of_head < worth ? of_head : worth;
}
// Whether a second launch adds parts (a cache without pages has none, whatever its table's width)
static bool joins(int64_t page, int64_t width, int64_t pieces) { return pieces > 0 && width * page > (kCutSteps - 1) * kChunkKeys; }
template <typename T, int BITS> static void chunk(const ChunkArgs &a, dim3 grid, dim3 join, hipStream_t st)
{
    const dim3 block(256);
    if (a.pieces == 0) {
        if (a.c.d <= 64) chunk_kernel<T, 64, 64, BITS, 0><<<grid, block, 0, st>>>(a);
        else if (a.c.d <= 96) chunk_kernel<T, 128, 96, BITS, 0><<<grid, block, 0, st>>>(a);
        else chunk_kernel<T, 128, 128, BITS, 0><<<grid, block, 0, st>>>(a);
        return;
    }
    switch (a.c.d) {
    case 16: chunk_kernel<T, 64, 64, BITS, 16><<<grid, block, 0, st>>>(a); break;
    case 32: chunk_kernel<T, 64, 64, BITS, 32><<<grid, block, 0, st>>>(a); break;
    case 48: chunk_kernel<T, 64, 64, BITS, 48><<<grid, block, 0, st>>>(a); break;
    case 64: chunk_kernel<T, 64, 64, BITS, 64><<<grid, block, 0, st>>>(a); break;
    case 80: chunk_kernel<T, 128, 96, BITS, 80><<<grid, block, 0, st>>>(a); break;
    case 96: chunk_kernel<T, 128, 96, BITS, 96><<<grid, block, 0, st>>>(a); break;
    case 112: chunk_kernel<T, 128, 128, BITS, 112><<<grid, block, 0, st>>>(a); break;
    default: chunk_kernel<T, 128, 128, BITS, 128><<<grid, block, 0, st>>>(a); break;
    }
    if (joins(a.c.page, a.width, a.pieces)) chunk_join_kernel<T><<<join, block, 0, st>>>(a);
}
}  // namespace s24_kv

using namespace s24_kv;

extern "C" int64_t s24_attn_chunk_workspace(const s24_kv_cache *cache, int64_t width, int64_t tokens, int64_t sequences, int64_t hq)
{
    if (cache == nullptr || cache->hkv <= 0 || cache->d <= 0 || cache->page <= 0 || width < 0 || tokens < 0 || sequences < 0 || hq <= 0 || hq % cache->hkv != 0) return 0;
    if (width * cache->page <= (kCutSteps - 1) * kChunkKeys) return 0;   // none is cut
    return chunk_pieces(cache, width, tokens, sequences, hq) * cache->hkv * kChunkRows * ((int64_t)sizeof(float2) + cache->d * 4);
}

extern "C" int s24_attn_chunk(const s24_kv_cache *cache, const s24_heads *Q, int64_t hq, const int32_t *cu, const int32_t *table, int64_t width, const int32_t *lengths,
                              int64_t sequences, int64_t tokens, float scale, int causal, const s24_heads *O, void *workspace, int64_t workspace_bytes, s24_dtype dt, void *stream)
{
    S24_TRY(check_cache(cache, dt));
    S24_REQUIRE(sequences >= 0 && sequences < INT32_MAX / 2 && tokens >= 0 && width >= 0 && width < INT32_MAX && hq > 0 && hq < 65536 && hq % cache->hkv == 0, S24_ERR_SHAPE);
    S24_REQUIRE(width * cache->page <= (int64_t)1 << 30 && tokens < INT32_MAX / 2 && tokens * (hq / cache->hkv) < INT32_MAX / 2, S24_ERR_SHAPE);
    S24_REQUIRE(width * cache->page * (hq / cache->hkv) < (int64_t)1 << 36, S24_ERR_SHAPE);   // (tiles of positions are counted in an int)
    S24_REQUIRE(scale > 0.0f && scale <= 3.0e38f, S24_ERR_SHAPE);
    S24_TRY(check_rows(Q, tokens, hq, cache->d, false));
    S24_TRY(check_rows(O, tokens, hq, cache->d, true));
    if (sequences == 0 || tokens == 0) return S24_OK;
    S24_REQUIRE(cu != nullptr && lengths != nullptr && (table != nullptr || width == 0), S24_ERR_NULL);
    const int64_t need = s24_attn_chunk_workspace(cache, width, tokens, sequences, hq);
    S24_REQUIRE(workspace != nullptr || need == 0, S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(cu, 4) && s24_aligned(table, 4) && s24_aligned(lengths, 4) && s24_aligned(workspace, 16), S24_ERR_ALIGN);
    S24_REQUIRE(workspace_bytes >= need, S24_ERR_SHAPE);
    const int64_t pieces = chunk_pieces(cache, width, tokens, sequences, hq), round = 2 * (int64_t)s24_cu_count() / cache->hkv, tiles = chunk_tiles(cache, tokens, sequences, hq), group = hq / cache->hkv;
    const int64_t groups = (pieces > tiles ? pieces : tiles) * cache->hkv;
    // About a thousand workgroups add the parts, each one to 64 rows.
    int sum_rows = 1;
    while (sum_rows < 64 && tokens * hq > 1024 * sum_rows) sum_rows *= 2;
    const int64_t join = most_tiles(tokens * group, tokens < sequences ? tokens : sequences, sum_rows) * cache->hkv;
    S24_REQUIRE(groups <= kMostGroups && (!joins(cache->page, cache->pages > 0 ? width : 0, pieces) || join <= kMostGroups), S24_ERR_SHAPE);
    ChunkArgs a{cache_of(cache), {static_cast<uint16_t *>(Q->data), Q->token, Q->head}, {static_cast<uint16_t *>(O->data), O->token, O->head}, cu, table, lengths,
                cache->pages > 0 ? width : 0, (int)sequences, (int)tokens, (int)group, causal != 0, (int)pieces, (int)(pieces < round ? pieces : round), sum_rows, scale};
    a.weights = static_cast<float2 *>(workspace);
    a.sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + pieces * cache->hkv * kChunkRows * sizeof(float2));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups), join_grid((unsigned)join);
    if (dt == S24_BF16) cache->bits == 16 ? chunk<uint16_t, 16>(a, grid, join_grid, st) : chunk<uint16_t, 8>(a, grid, join_grid, st);
    else cache->bits == 16 ? chunk<s24_half, 16>(a, grid, join_grid, st) : chunk<s24_half, 8>(a, grid, join_grid, st);
    return s24_launch_status();
}
