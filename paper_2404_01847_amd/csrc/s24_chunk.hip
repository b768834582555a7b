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
    int sequences, tokens, hq, group, causal, parts;
    bool mix;          // order of the tiles: by length alone, or sequence by sequence
    float scale;
    float2 *weights;   // [parts][tokens][hq]: reference and sum
    float *sums;       // [parts][tokens][hq][d]
};
constexpr int kChunkRows = 128, kChunkKeys = 64;
__device__ __forceinline__ Span keys_of(const ChunkArgs &a, int i) { return {0, min(max(a.lengths[i], 0), (int)(a.width << a.c.shift))}; }
// The workgroup's tile: a sequence, and which of its tiles, the last ones first
__device__ __forceinline__ bool find_chunk(const ChunkArgs &a, int t, int lane, int &sequence, int &tile)
{
    int at;
    auto of = [&](int i) {
        const int n = (int)(((int64_t)span(a.cu, i, a.tokens).count * a.group + kChunkRows - 1) / kChunkRows), keys = (int)(((int64_t)keys_of(a, i).count * a.group + kChunkRows - 1) / kChunkRows);
        return a.causal ? Lengths{n, max(keys, n), INT32_MAX} : Lengths{n, INT32_MAX, max(keys, 1)};
    };
    const int64_t most = max((int64_t)a.tokens, a.width << a.c.shift) * a.group / kChunkRows + 1;
    if (!find_by_length(a.mix, a.sequences, t, (int)most, lane, sequence, at, of)) return false;
    tile = of(sequence).tiles - 1 - at;
    return true;
}

// Keys of a tile in LDS: piece c of a row at slot c ^ flip.  The 16 rows of an operand are four of each sixteen positions, of which the LDS takes those of lanes 0-3 and 12-15
// of one piece together with those of lanes 4-11 of the next in a cycle.
template <int D> __device__ __forceinline__ int flip(int row) { return D == 128 ? ((row & 3) | (row >> 4 & 1) << 2) << 1 : ((row >> 1 & 1) | (row >> 4 & 1) << 1) << 1; }

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
            const int row = i * (512 / D) + lane / (D / 8), piece = (lane % (D / 8)) ^ flip<D>(16 * wave + row);
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
    __device__ __forceinline__ void init(const Cache &c, int wave_, int lane_)
    {
        wave = wave_, lane = lane_;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = 64 * i + lane;
            from_k[i] = (uint32_t)((at / (D / 16)) * c.d + 16 * min(at % (D / 16), (c.d >> 4) - 1));
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
            const int at = 64 * i + lane, row = 16 * wave + at / (D / 16), piece = 2 * (at % (D / 16));
            lds_byte *const to = tk + row * 2 * D;
            lds_store(to + ((piece ^ flip<D>(row)) << 4), halves(k[i].x, k[i].y));
            lds_store(to + (((piece + 1) ^ flip<D>(row)) << 4), halves(k[i].z, k[i].w));
            lds_store(tv + (2 * wave * D + at) * 16, halves(v[i].x, v[i].y));
            lds_store(tv + ((2 * wave + 1) * D + at) * 16, halves(v[i].z, v[i].w));
        }
        if (lane < 32) steps[(lane >> 4) * kChunkKeys + 16 * wave + (lane & 15)] = lane < 16 || (lane & 15) < left ? step : 0.0f;
    }
};

// D: values of a tile's row; E: values that the products go over
template <typename T, int D, int E, int BITS>
__global__ __launch_bounds__(256, 2) void chunk_kernel(const ChunkArgs a)
{
    using M = typename std::conditional<BITS == 8, s24_half, T>::type;
    using Num = s24_num<T>;
    constexpr int BK = kChunkKeys, TILE = BK * 2 * D;
    __shared__ __align__(16) unsigned char lds_k[2][TILE], lds_v[2][TILE];
    __shared__ __align__(16) float steps[2][BITS == 8 ? 2 * BK : 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const Unit unit = unit_of(blockIdx.x, a.c.hkv, a.parts);
    const int kv = unit.head;
    int sequence, index;
    if (!find_chunk(a, unit.tile, lane, sequence, index)) return;
    Queries s_;
    s_.init(span(a.cu, sequence, a.tokens), keys_of(a, sequence), a.group, a.causal, index, kChunkRows, 32 * wave);
    const int length = s_.k.count, all_tiles = s_.seen > 0 ? (s_.seen + BK - 1) / BK : 0;
    const int begin = (int)((int64_t)all_tiles * unit.part / a.parts), tiles = (int)((int64_t)all_tiles * (unit.part + 1) / a.parts);

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
        if constexpr (BITS == 8) {   // scaled by a power of two into what binary16 holds
            float most = 0.0f;
#pragma unroll
            for (int k = 0; k < E / 32; ++k)
                for (const uint32_t x : {q[j][k].x, q[j][k].y, q[j][k].z, q[j][k].w}) most = fmaxf(most, fmaxf(fabsf(Num::lo(x)), fabsf(Num::hi(x))));
            most = column_max(most);
            const int e = most > 0.0f ? ilogbf(most) : 0;
            auto scaled = [&](uint32_t x) { return pack2<s24_half>(ldexpf(Num::lo(x), -e), ldexpf(Num::hi(x), -e)); };
#pragma unroll
            for (int k = 0; k < E / 32; ++k) q[j][k] = make_uint4(scaled(q[j][k].x), scaled(q[j][k].y), scaled(q[j][k].z), scaled(q[j][k].w));
            c[j] = ldexpf(c[j], e);
        }
    }
    float m[2] = {-1e30f, -1e30f}, l[2] = {0.0f, 0.0f};
    float rise = BITS == 8 ? -100.0f : 0.0f, wide = 0x1p-100f;   // the reference's part from the steps of V, which are at most `wide`
    f32x4 o[E / 16][2];
#pragma unroll
    for (int n = 0; n < E / 16; ++n) o[n][0] = o[n][1] = f32x4{};

    Sixteen<D, BITS> sixteen;
    sixteen.init(a.c, wave, lane);
    const int *table = a.table + sequence * a.width;
    // Where the wave's positions of tile t are, in tokens of one head.  (Those past the sequence's end are its last ones again.)
    auto page_of = [&](int t) {
        const int pos = min(t * BK + 16 * wave, (length - 1) & ~15);
        return min((uint32_t)table[pos >> a.c.shift], (uint32_t)a.c.pages - 1);
    };
    auto place = [&](int t, uint32_t id) {
        const int pos = min(t * BK + 16 * wave, (length - 1) & ~15);
        return (((int64_t)id * a.c.hkv + kv) << a.c.shift) + (pos & (a.c.page - 1));
    };
    uint32_t id = 0;   // of the next tile
    if (begin < tiles) {
        sixteen.start(a.c, place(begin, page_of(begin)), (lds_byte *)lds_k[begin & 1], (lds_byte *)lds_v[begin & 1], steps[begin & 1]);
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
                    const uint4 f = lds_load(tk + row * 2 * D + (((4 * k + g) ^ flip<D>(row)) << 4));
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
            if (__any(top[0] > m[0] - rise + kGrowth || top[1] > m[1] - rise + kGrowth || (BITS == 8 && step > wide))) {
                if (BITS == 8) {
                    step = column_max(step);
                    if (step > wide) wide = 2.0f * step;
                }
                const float lift = BITS == 8 ? __builtin_amdgcn_logf(wide) : 0.0f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float now = fmaxf(m[j] - rise, column_max(top[j])) + lift, shrink = __builtin_amdgcn_exp2f(m[j] - now);
                    m[j] = now, l[j] *= shrink;
#pragma unroll
                    for (int n = 0; n < E / 16; ++n) o[n][j] *= shrink;
                }
                rise = lift;
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
                    o[n][0] = mma<M>(f, p[u][0], o[n][0]);
                    o[n][1] = mma<M>(f, p[u][1], o[n][1]);
                }
        }
        if (t + 1 < tiles) sixteen.finish((lds_byte *)lds_k[other], (lds_byte *)lds_v[other], steps[other], length - (t + 1) * BK - 16 * wave);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = 32 * wave + 16 * j + col;
        const float sum = column_sum(l[j]), inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (s_.row0 + row >= s_.rows) continue;
        const Queries::Row of = s_.row(a.group, kv, row);
        if (a.parts == 1) {
            uint16_t *out = a.o.p + of.token * a.o.token + of.head * a.o.head;
#pragma unroll
            for (int n = 0; n < E / 16; n += 4) {   // of four such pieces of a row a lane gets one whole: lines are written with few stores
                uint32_t x[4], y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 v = n + i < E / 16 ? o[n + i < E / 16 ? n + i : 0][j] * inverse : f32x4{};
                    x[i] = pack2<T>(v[0], v[1]), y[i] = pack2<T>(v[2], v[3]);
                }
                transpose_rows(x), transpose_rows(y);
                const int at = 16 * (n + g);
                if (at >= a.c.d) continue;
                *reinterpret_cast<uint4 *>(out + at) = make_uint4(x[0], y[0], x[1], y[1]);
                *reinterpret_cast<uint4 *>(out + at + 8) = make_uint4(x[2], y[2], x[3], y[3]);
            }
        } else {
            const int64_t at = (unit.part * (int64_t)a.tokens + of.token) * a.hq + of.head;
#pragma unroll
            for (int n = 0; n < E / 16; ++n)
                if (16 * n < a.c.d) *reinterpret_cast<f32x4 *>(a.sums + at * a.c.d + 16 * n + 4 * g) = o[n][j];
            if (g == 0) a.weights[at] = make_float2(m[j], sum);
        }
    }
}

// O from the sums of the parts
template <typename T>
__global__ __launch_bounds__(256) void chunk_join_kernel(const ChunkArgs a)
{
    Joined j;
    if (!join_rows(a.cu, a.sequences, a.tokens, a.hq, j)) return;
    const int d = a.c.d, quads = d >> 2;
    const int64_t step = (int64_t)a.tokens * a.hq;
    for (int item = threadIdx.x; item < j.rows * quads; item += 256) {
        const int row = item / quads, i = 4 * (item - row * quads);
        const int64_t t = j.first + row, at = t * a.hq + j.head;
        float m = -1e30f, l = 0.0f;
        for (int p = 0; p < a.parts; ++p) m = fmaxf(m, a.weights[at + p * step].x);
        f32x4 x = {};
        for (int p = 0; p < a.parts; ++p) {
            const float2 w = a.weights[at + p * step];
            const float f = __builtin_amdgcn_exp2f(w.x - m);
            l = fmaf(w.y, f, l), x += *reinterpret_cast<const f32x4 *>(a.sums + (at + p * step) * d + i) * f;
        }
        x *= l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2 *>(a.o.p + t * a.o.token + j.head * a.o.head + i) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    }
}

// ------------------------------------------------------------------ host
static int64_t chunk_groups(int64_t tokens, int64_t sequences, int64_t hq, int64_t hkv)
{
    return (tokens * (hq / hkv) / kChunkRows + (tokens < sequences ? tokens : sequences)) * hkv;
}
// Parts of the positions, by the estimate of the forward pass; the host knows of the lengths only what the table holds
static int chunk_parts(const s24_kv_cache *c, int64_t width, int64_t tokens, int64_t sequences, int64_t hq)
{
    return parts_for((double)chunk_groups(tokens, sequences, hq, c->hkv), (double)(width * c->page) / kChunkKeys, 1.0, c->d <= 64 ? 1.05 : 1.5,
                     (double)tokens * (double)hq * (double)c->d * 4.0);
}
static int64_t weight_bytes(int64_t tokens, int64_t hq) { return (tokens * hq * (int64_t)sizeof(float2) + 15) / 16 * 16; }

template <typename T, int BITS> static void chunk(const ChunkArgs &a, dim3 grid, dim3 join, hipStream_t st)
{
    const dim3 block(256);
    if (a.c.d <= 64) chunk_kernel<T, 64, 64, BITS><<<grid, block, 0, st>>>(a);
    else if (a.c.d <= 96) chunk_kernel<T, 128, 96, BITS><<<grid, block, 0, st>>>(a);
    else chunk_kernel<T, 128, 128, BITS><<<grid, block, 0, st>>>(a);
    if (a.parts > 1) chunk_join_kernel<T><<<join, block, 0, st>>>(a);
}
}  // namespace s24_kv

using namespace s24_kv;

extern "C" int64_t s24_attn_chunk_workspace(const s24_kv_cache *cache, int64_t width, int64_t tokens, int64_t sequences, int64_t hq)
{
    if (cache == nullptr || cache->hkv <= 0 || cache->d <= 0 || cache->page <= 0 || width < 0 || tokens < 0 || sequences < 0 || hq <= 0 || hq % cache->hkv != 0) return 0;
    const int64_t parts = chunk_parts(cache, width, tokens, sequences, hq);
    return parts > 1 ? parts * (weight_bytes(tokens, hq) + tokens * hq * cache->d * 4) : 0;
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
    const int parts = chunk_parts(cache, width, tokens, sequences, hq);
    const int64_t groups = chunk_groups(tokens, sequences, hq, cache->hkv) * parts, join = most_tiles(tokens, sequences, kJoinRows) * hq;
    S24_REQUIRE(groups <= kMostGroups && join <= kMostGroups, S24_ERR_SHAPE);
    ChunkArgs a{cache_of(cache), {static_cast<uint16_t *>(Q->data), Q->token, Q->head}, {static_cast<uint16_t *>(O->data), O->token, O->head}, cu, table, lengths,
                cache->pages > 0 ? width : 0, (int)sequences, (int)tokens, (int)hq, (int)(hq / cache->hkv), causal != 0, parts};
    a.mix = sequences > 1, a.scale = scale;
    a.weights = static_cast<float2 *>(workspace);
    a.sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + parts * weight_bytes(tokens, hq));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups), join_grid((unsigned)join);
    if (dt == S24_BF16) cache->bits == 16 ? chunk<uint16_t, 16>(a, grid, join_grid, st) : chunk<uint16_t, 8>(a, grid, join_grid, st);
    else cache->bits == 16 ? chunk<s24_half, 16>(a, grid, join_grid, st) : chunk<s24_half, 8>(a, grid, join_grid, st);
    return s24_launch_status();
}
