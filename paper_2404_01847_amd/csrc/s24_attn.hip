// Attention over packed sequences, forward and backward (the training step's other half, and the reading of prompts).
//
// S_ij = c q_i.k_j over the visible pairs, P = softmax of its rows, O = P V.  Forward: one pass over the keys with the running maximum and sum
// of each row; S^T is formed with the keys as rows, so that a lane holds one query's scores, the row statistics need no exchange between lanes
// but a rare one, and the rounded P is the second product's operand as it lies in the registers.
// Backward, from lse_i = log sum_j exp S_ij and delta_i = dO_i.O_i (of O with what its rounding took away, which
// the forward pass leaves in a byte for each value):  P_ij = exp(S_ij - lse_i),  dV = P^T dO,  dS_ij = P_ij (dO_i.v_j - delta_i),
// dQ = c dS K,  dK = c dS^T Q.
// Sums run over queries for dK and dV and over keys for dQ: two parts, each of which forms S and dO V^T for itself (7 products instead of 5, and two more
// for the second halves of dS).  One kernel would have to add to dQ from many workgroups, in an order that no two runs share.
// What bounds it: the matrix instructions and the vector instructions on the scores, which a compute unit runs at the same time only in part.  (Two waves of nothing
// but 16x16x32 instructions take 8.1 ns for each on a SIMD; with four fma to each 12.2.)  8192 tokens, 64 heads on 8 of 128: 1.00 ms for O (1.10 PFLOP/s; a library's plain
// products of 8192 x 8192 x 8192 reach 1.37 to 1.58), matrix cores 53 % busy; 1.81 ms for dQ, 57 %; 2.39 ms for dK and dV, 55 %.
#include "s24_attn.h"

#include <math.h>

namespace s24_attn {

struct Rows { const uint16_t *p; int64_t token, head; };   // element (t, h, i) at p + t*token + h*head + i
struct Out { uint16_t *p; int64_t token, head; };
struct Problem {
    Rows q, k, v, o, dO;
    Out out, dq, dk, dv;
    int8_t *rest;          // [tokens_q][hq][d]: what the rounding of O took away; or NULL
    float *lse;            // [hq][tokens_q]
    float2 *stats;         // [hq][tokens_q], of the backward pass: what a row's exponents are taken from, and delta
    // Where a kernel's workgroups are few, what a tile sums over is cut into parts, whose sums another kernel adds
    struct Cut {
        int parts;
        float *sums;       // [parts][tokens][heads][values]
    } by_query, by_key;    // O or dQ; dK and dV
    float2 *weights;       // [parts][tokens_q][hq], of the forward pass: reference and sum
    unsigned key_blocks;   // workgroups for dK and dV in a launch that has those for dQ after them
    const int *cu_q, *cu_k;
    int sequences, tokens_q, tokens_k, hq, group, d, causal;
    bool mix_queries, mix_keys;   // order of the tiles of queries, of keys: by length alone, or sequence by sequence
    float scale;
};

// The workgroup's tile: a sequence, and which of its tiles.  When causal the last ones see the most keys.
__device__ __forceinline__ bool find_queries(const Problem &a, int rows, int t, int lane, int &sequence, int &tile)
{
    int at;
    auto of = [&](int i) {
        const int n = (span(a.cu_q, i, a.tokens_q).count * a.group + rows - 1) / rows, keys = (span(a.cu_k, i, a.tokens_k).count * a.group + rows - 1) / rows;
        return a.causal ? Lengths{n, max(keys, n), INT32_MAX} : Lengths{n, INT32_MAX, max(keys, 1)};
    };
    if (!find_by_length(a.mix_queries, a.sequences, t, max(a.tokens_q, a.tokens_k) * a.group / rows + 1, lane, sequence, at, of)) return false;
    tile = of(sequence).tiles - 1 - at;
    return true;
}
// Of `rows` keys: when causal the first ones are seen by the most queries, by all of them as far as the queries have keys before them.
__device__ __forceinline__ bool find_keys(const Problem &a, int rows, int t, int lane, int &sequence, int &tile)
{
    return find_by_length(a.mix_keys, a.sequences, t, max(a.tokens_q, a.tokens_k) / rows + 1, lane, sequence, tile, [&](int i) {
        const int n = (span(a.cu_k, i, a.tokens_k).count + rows - 1) / rows, queries = (span(a.cu_q, i, a.tokens_q).count + rows - 1) / rows;
        return Lengths{n, a.causal ? n : INT32_MAX, max(queries, 1)};
    });
}

// ------------------------------------------------------------------ forward
// Four waves of 32 rows.  Keys and values in tiles of 64, two of them in LDS: the next one is copied during the work on this one, with one barrier a tile.
// (Instructions of 32 x 32 x 16 in place of 16 x 16 x 32 are half as many, but the products wait more: 4 x 4096 tokens of 32 heads of 128 578 us for 543, 8 x 1024
// of 12 heads of 64, both passes, 112 for 108.  Keys and values in one array of LDS cost 5 %: the compiler then
// cannot tell the copies of the one from the reads of the other.
// Tiles of 32 keys with three waves to a SIMD, and tiles of 64 rows, were no faster on operands that come from memory.)
template <int D> struct Forward {
    static constexpr int BK = 64, TILE = BK * 2 * D;
};

// D: values of a tile's row; E: values that the products go over.  (Heads of 96 in tiles of 128 by products of 128: two sequences of 4096 tokens, 16 heads on 4, 139 us forward
// and 565 backward; of 96 120 and 477.  Heads of 80 137 and 554, and 118 and 471.  One sequence of 8192, heads of 96: 257 and 1065, and 217 and 896.)
template <typename T, int D, int E>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(const Problem a)
{
    using C = Forward<D>;
    constexpr int BQ = 128, NI = C::BK / 16;   // rows of a workgroup, of 16 keys in a tile
    __shared__ __align__(16) unsigned char lds_k[2][C::TILE], lds_v[2][C::TILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const Unit unit = unit_of(blockIdx.x, a.hq / a.group, a.by_query.parts);
    const int kv = unit.head;
    int sequence, index;
    if (!find_queries(a, BQ, unit.tile, lane, sequence, index)) return;
    Queries s_;
    s_.init(span(a.cu_q, sequence, a.tokens_q), span(a.cu_k, sequence, a.tokens_k), a.group, a.causal, index, BQ, 32 * wave);
    const Span sk = s_.k;
    const int all_tiles = s_.seen > 0 ? (s_.seen + C::BK - 1) / C::BK : 0;
    const int begin = (int)((int64_t)all_tiles * unit.part / a.by_query.parts), tiles = (int)((int64_t)all_tiles * (unit.part + 1) / a.by_query.parts);

    uint4 q[2][E / 32];
    int last[2];   // that a row sees
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const Queries::Row of = s_.row(a.group, kv, 32 * wave + 16 * j + col);
        const uint16_t *row = a.q.p + of.token * a.q.token + of.head * a.q.head;
        last[j] = a.causal ? min(sk.count - 1, of.at + s_.ahead) : sk.count - 1;
#pragma unroll
        for (int k = 0; k < E / 32; ++k)
            q[j][k] = 32 * k + 8 * g < a.d ? *reinterpret_cast<const uint4 *>(row + 32 * k + 8 * g) : make_uint4(0, 0, 0, 0);
    }
    const float c = a.scale * kLog2e;
    float m[2] = {-1e30f, -1e30f}, l[2] = {0.0f, 0.0f};
    f32x4 o[E / 16][2];
#pragma unroll
    for (int n = 0; n < E / 16; ++n) o[n][0] = o[n][1] = f32x4{};

    const uint16_t *keys = a.k.p + sk.first * a.k.token + kv * a.k.head, *values = a.v.p + sk.first * a.v.token + kv * a.v.head;
    Copy<D, C::BK, 4> ck, cv;
    ck.init(wave, lane, (int)a.k.token * 2, a.d), cv.init(wave, lane, (int)a.v.token * 2, a.d);
    auto copy = [&](int t) {
        const int left = sk.count - t * C::BK;
        if (left < C::BK) ck.offsets(left), cv.offsets(left);
        ck.start(keys + (int64_t)t * C::BK * a.k.token, (lds_byte *)lds_k[t & 1]);
        cv.start(values + (int64_t)t * C::BK * a.v.token, (lds_byte *)lds_v[t & 1]);
    };
    if (begin < tiles) copy(begin);
    for (int t = begin; t < tiles; ++t) {
        wait_and_barrier<0>();
        if (t + 1 < tiles) copy(t + 1);
        const int k0 = t * C::BK;
        if (k0 >= s_.wave_seen) continue;
        const lds_byte *tk = (const lds_byte *)lds_k[t & 1], *tv = (const lds_byte *)lds_v[t & 1];
        f32x4 s[NI][2];
#pragma unroll
        for (int i = 0; i < NI; ++i) s[i][0] = s[i][1] = f32x4{};
#pragma unroll
        for (int k = 0; k < E / 32; ++k)
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint4 f = rows<D>(tk, 16 * i, k, lane);
                s[i][0] = mma<T>(f, q[0][k], s[i][0]);
                s[i][1] = mma<T>(f, q[1][k], s[i][1]);
            }
        if (D == 128) reads_ahead<NI, 2 * NI, E / 32>();
        if (k0 + C::BK > s_.wave_all) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[i][j][r] = k0 + 16 * i + 4 * g + r <= last[j] ? s[i][j][r] : -INFINITY;
        }
        float top[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            top[j] = s[0][j][0];
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) top[j] = fmaxf(top[j], s[i][j][r]);
            top[j] *= c;
        }
        if (__any(top[0] > m[0] + kGrowth || top[1] > m[1] + kGrowth)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float now = fmaxf(m[j], column_max(top[j])), shrink = __builtin_amdgcn_exp2f(m[j] - now);
                m[j] = now, l[j] *= shrink;
#pragma unroll
                for (int n = 0; n < E / 16; ++n) o[n][j] *= shrink;
            }
        }
        uint4 p[NI / 2][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c, -m[j]));
                    l[j] += s[i][j][r];
                }
#pragma unroll
            for (int u = 0; u < NI / 2; ++u) p[u][j] = operand<T>(s[2 * u][j], s[2 * u + 1][j]);
        }
#pragma unroll
        for (int u = 0; u < NI / 2; ++u)
#pragma unroll
            for (int n = 0; n < E / 16; ++n) {
                const uint4 f = columns<D>(tv, 32 * u, n, lane);
                o[n][0] = mma<T>(f, p[u][0], o[n][0]);
                o[n][1] = mma<T>(f, p[u][1], o[n][1]);
            }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = 32 * wave + 16 * j + col;
        const float sum = column_sum(l[j]), inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (s_.row0 + row >= s_.rows) continue;
        const Queries::Row of = s_.row(a.group, kv, row);
        const int64_t token = of.token;
        const int head = of.head;
        if (a.by_query.parts == 1) {
            uint16_t *out = a.out.p + token * a.out.token + head * a.out.head;
            int8_t *rest = a.rest + (token * a.hq + head) * a.d;
#pragma unroll
            for (int n = 0; n < E / 16; n += 4) {   // of four such pieces of a row a lane gets one whole: lines are written with few stores
                uint32_t x[4], y[4], left[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 v = n + i < E / 16 ? o[n + i < E / 16 ? n + i : 0][j] * inverse : f32x4{};
                    x[i] = pack2<T>(v[0], v[1]), y[i] = pack2<T>(v[2], v[3]);
                    left[i] = a.rest != nullptr ? four_left<T>(v, make_uint2(x[i], y[i])) : 0;
                }
                transpose_rows(x), transpose_rows(y);
                if (a.rest != nullptr) transpose_rows(left);
                const int at = 16 * (n + g);
                if (at >= a.d) continue;
                *reinterpret_cast<uint4 *>(out + at) = make_uint4(x[0], y[0], x[1], y[1]);
                *reinterpret_cast<uint4 *>(out + at + 8) = make_uint4(x[2], y[2], x[3], y[3]);
                if (a.rest != nullptr) *reinterpret_cast<uint4 *>(rest + at) = make_uint4(left[0], left[1], left[2], left[3]);
            }
            if (a.lse != nullptr && g == 0) a.lse[(int64_t)head * a.tokens_q + token] = sum == 0.0f ? -INFINITY : (m[j] + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
            const int64_t at = (unit.part * (int64_t)a.tokens_q + token) * a.hq + head;
#pragma unroll
            for (int n = 0; n < E / 16; ++n)
                if (16 * n < a.d) *reinterpret_cast<f32x4 *>(a.by_query.sums + at * a.d + 16 * n + 4 * g) = o[n][j];
            if (g == 0) a.weights[at] = make_float2(m[j], sum);
        }
    }
}

// O and lse from the sums of the parts
template <typename T>
__global__ __launch_bounds__(256) void attn_fwd_join_kernel(const Problem a)
{
    Joined j;
    if (!join_rows(a.cu_q, a.sequences, a.tokens_q, a.hq, j)) return;
    const int quads = a.d >> 2;
    const int64_t step = (int64_t)a.tokens_q * a.hq;
    for (int item = threadIdx.x; item < j.rows * quads; item += 256) {
        const int row = item / quads, i = 4 * (item - row * quads);
        const int64_t t = j.first + row, at = t * a.hq + j.head;
        float m = -1e30f, l = 0.0f;
        for (int p = 0; p < a.by_query.parts; ++p) m = fmaxf(m, a.weights[at + p * step].x);
        f32x4 x = {};
        for (int p = 0; p < a.by_query.parts; ++p) {
            const float2 w = a.weights[at + p * step];
            const float f = __builtin_amdgcn_exp2f(w.x - m);
            l = fmaf(w.y, f, l), x += *reinterpret_cast<const f32x4 *>(a.by_query.sums + (at + p * step) * a.d + i) * f;
        }
        x *= l == 0.0f ? 0.0f : 1.0f / l;
        const uint2 stored = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
        *reinterpret_cast<uint2 *>(a.out.p + t * a.out.token + j.head * a.out.head + i) = stored;
        if (a.rest != nullptr) *reinterpret_cast<uint32_t *>(a.rest + at * a.d + i) = four_left<T>(x, stored);
        if (i == 0 && a.lse != nullptr) a.lse[(int64_t)j.head * a.tokens_q + t] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

// ------------------------------------------------------------------ backward
// P is formed times 2^kUp, from lse - kUp: exp2 gives zero for what fp32 has no normal number for, and binary16 holds weights below 2^-14 with fewer bits.
// The factor goes through dS to the end of the sums.  dS is of any size (about dO's over a row's length, or thousands of dO's), for which binary16 has no room: there it
// is taken times a power of two more, `Moving`.
template <typename T> struct Lift;
template <> struct Lift<uint16_t> { static constexpr float kUp = 32.0f, kBack = 0x1p-32f; static constexpr bool kMoves = false; };
template <> struct Lift<s24_half> { static constexpr float kUp = 15.0f, kBack = 0x1p-15f; static constexpr bool kMoves = true; };

// The factor of a column of dS (a query's in dQ, a key's in dK; alike in its four lanes).  It is set such that the column's largest value so far is between 2^7 and 2^8, and again when one
// reaches 2^15: the pair of operands then loses nothing above 2^-32 of the largest, and nothing becomes infinite.  Of visible pairs only: what a column does not see does not
// move it.  (Without it dO about 1e-3 and 4096 keys give a dQ four times as far from 64 bits as its own rounding is, and dO of 12000 NaN.  The watch costs 4 to 6 %: gradients of 8192
// tokens in binary16, 64 heads on 8 of 128, 4.09 ms without it and 4.27 with, 16 on 4 of 64 615 us and 650, of 8 x 1024 tokens of 12 heads of 64 82 and 86.  A factor from the first
// tile alone, with the tile done again where it proves too large, costs 3 % of the largest and 8 of the smallest.)
struct Moving {
    float by = 0x1p24f;
    __device__ __forceinline__ float back() const { return 1.0f / by; }
    // By which the sums and values so far are taken on: `most` is the largest of this lane's values
    __device__ __forceinline__ float step(float most)
    {
        most = column_max(most);
        if (!(most >= 0x1p15f) || most == INFINITY) return 1.0f;
        const float f = ldexpf(1.0f, 7 - ilogbf(most));
        by *= f;
        return f;
    }
};
__device__ __forceinline__ float largest(float most, f32x4 x)
{
    return fmaxf(fmaxf(fmaxf(fmaxf(most, fabsf(x[0])), fabsf(x[1])), fabsf(x[2])), fabsf(x[3]));
}

// dK and dV of 128 keys of a key-value head, four waves of 32: over the query heads of the group and their queries, 32 at a time.
// S has the queries as rows, so that P and dS are, as they lie, the operands that contract over the queries.  A step has 80 matrix instructions of a wave (heads of
// 128), 28 reads of 16 bytes and 32 transposed ones; at two waves to a SIMD it takes 1.9 us, of which the matrix instructions are 1.1.
template <int D> struct Backward {
    static constexpr int BK = 128, BQ = 32, TILE = BQ * 2 * D, STAGE = 2 * TILE + 8 * BQ, VALUES = BK * 2 * D;   // a stage: queries, gradients, row statistics
};
// tv, stages: C::VALUES and two times C::STAGE bytes of LDS
template <typename T, int D, int E> __device__ __forceinline__ void dkv_tile(const Problem &a, unsigned block, lds_byte *tv, lds_byte *stages)
{
    using C = Backward<D>;
    using L = Lift<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int hkv = a.hq / a.group;
    const Unit unit = unit_of(block, hkv, a.by_key.parts);
    const int kv = unit.head, part = unit.part;
    int sequence, index;
    if (!find_keys(a, C::BK, unit.tile, lane, sequence, index)) return;
    const Span sq = span(a.cu_q, sequence, a.tokens_q), sk = span(a.cu_k, sequence, a.tokens_k);
    const int k0 = index * C::BK, wk0 = k0 + 32 * wave;
    const int ahead = sk.count - sq.count;
    const int first = a.causal ? max(0, k0 - ahead) / C::BQ : 0;                // query tiles
    const int each = max(0, (sq.count + C::BQ - 1) / C::BQ - first);
    // the steps of all heads of the group, and of them this part's
    const int64_t all_steps = (int64_t)each * a.group;
    const int begin = (int)(all_steps * part / a.by_key.parts), steps = (int)(all_steps * (part + 1) / a.by_key.parts) - begin;

    // The keys' fragments stay in registers, the values' come from LDS: with both, two waves would not fit a SIMD (8192 tokens, 64 heads on 8 of 128: 3.6 ms
    // with both in registers, 2.0 so, before dS went in two parts).
    uint4 fk[2][E / 32];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t t = sk.first + min(wk0 + 16 * j + col, sk.count - 1);
#pragma unroll
        for (int k = 0; k < E / 32; ++k) {
            const int i = 32 * k + 8 * g;
            fk[j][k] = i < a.d ? *reinterpret_cast<const uint4 *>(a.k.p + t * a.k.token + kv * a.k.head + i) : make_uint4(0, 0, 0, 0);
        }
    }
    {
        Copy<D, C::BK, 4> cv;
        cv.init(wave, lane, (int)a.v.token * 2, a.d);
        cv.offsets(min(sk.count - k0, C::BK));
        cv.start(a.v.p + (int64_t)(sk.first + k0) * a.v.token + kv * a.v.head, tv);
        if (a.d < D) {   // past the head's last value: zeros, of which no gradient row makes anything else
            wait_and_barrier<0>();
            for (int i = threadIdx.x; i < C::BK * (D / 8); i += 256)
                if (8 * (i % (D / 8)) >= a.d) lds_store(tv + piece<D>(i / (D / 8), i % (D / 8)), make_uint4(0, 0, 0, 0));
        }
    }
    f32x4 dk[E / 16][2], dv[E / 16][2];
#pragma unroll
    for (int n = 0; n < E / 16; ++n) dk[n][0] = dk[n][1] = dv[n][0] = dv[n][1] = f32x4{};
    const float c = a.scale * kLog2e;
    Moving moving[2];

    Copy<D, C::BQ, 4> cq, cdo;
    cq.init(wave, lane, (int)a.q.token * 2, a.d), cdo.init(wave, lane, (int)a.dO.token * 2, a.d);
    int next_head = kv * a.group + (each > 0 ? begin / each : 0), next_tile = first + (each > 0 ? begin % each : 0), buffer = 0;
    int qt = next_tile;
    auto copy = [&](int stage) {
        const int left = sq.count - next_tile * C::BQ;
        cq.offsets(min(left, C::BQ)), cdo.offsets(min(left, C::BQ));
        const int64_t t = sq.first + next_tile * C::BQ;
        lds_byte *to = stages + stage * C::STAGE;
        cq.start(a.q.p + t * a.q.token + next_head * a.q.head, to);
        cdo.start(a.dO.p + t * a.dO.token + next_head * a.dO.head, to + C::TILE);
        if (wave == 0) buffer_to_lds<4>(buffer_of(a.stats + ((int64_t)next_head * a.tokens_q + t)), (lds_ptr)(to + 2 * C::TILE), 4u * (uint32_t)min(lane, 2 * left - 2 + (lane & 1)));
        if (++next_tile == first + each) next_tile = first, ++next_head;
    };
    if (steps > 0) copy(0);
    for (int step = 0; step < steps; ++step) {
        wait_and_barrier<0>();
        if (step + 1 < steps) copy(buffer ^ 1);
        const int q0 = qt * C::BQ, now = buffer;
        buffer ^= 1;
        if (++qt == first + each) qt = first;
        if (wk0 >= sk.count || (a.causal && q0 + C::BQ - 1 + ahead < wk0)) continue;   // no query of the tile sees a key of the wave
        const lds_byte *tq = stages + now * C::STAGE, *tdo = tq + C::TILE, *stats = tdo + C::TILE;
        f32x4 s[2][2], dp[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = dp[i][0] = dp[i][1] = f32x4{};
#pragma unroll
        for (int k = 0; k < E / 32; ++k) {
            uint4 fv[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) fv[j] = rows<D>(tv, 32 * wave + 16 * j, k, lane);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 x = rows<D>(tq, 16 * i, k, lane), y = rows<D>(tdo, 16 * i, k, lane);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[i][j] = mma<T>(x, fk[j][k], s[i][j]);
                    dp[i][j] = mma<T>(y, fv[j], dp[i][j]);
                }
            }
        }
        const bool all = q0 + C::BQ <= sq.count && wk0 + 32 <= sk.count && (!a.causal || wk0 + 31 <= q0 + ahead);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x4 lse, delta;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float4 two = __builtin_bit_cast(float4, lds_load(stats + 8 * (16 * i + 4 * g + 2 * r)));
                lse[2 * r] = two.x, delta[2 * r] = two.y, lse[2 * r + 1] = two.z, delta[2 * r + 1] = two.w;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c, -lse[r]));
                    dp[i][j][r] = (L::kMoves ? s[i][j][r] * moving[j].by : s[i][j][r]) * (dp[i][j][r] - delta[r]);
                }
        }
        if (!all) {   // whatever stands in rows past the last, nothing of it stays
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int key = wk0 + 16 * j + col, lo = key >= sk.count ? sq.count : a.causal ? key - ahead : 0;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int query = q0 + 16 * i + 4 * g + r;
                        const bool visible = (query >= lo) & (query < sq.count);
                        s[i][j][r] = visible ? s[i][j][r] : 0.0f, dp[i][j][r] = visible ? dp[i][j][r] : 0.0f;
                    }
            }
        }
        if constexpr (L::kMoves) {
            float most[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) most[j] = largest(largest(0.0f, dp[0][j]), dp[1][j]);
            if (__any(most[0] >= 0x1p15f || most[1] >= 0x1p15f)) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float f = moving[j].step(most[j]);
                    dp[0][j] *= f, dp[1][j] *= f;
#pragma unroll
                    for (int n = 0; n < E / 16; ++n) dk[n][j] *= f;
                }
            }
        }
        uint4 p[2], ds[2], lo[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) p[j] = operand<T>(s[0][j], s[1][j]), ds[j] = operand<T>(dp[0][j], dp[1][j]), lo[j] = rest<T>(ds[j], dp[0][j], dp[1][j]);
#pragma unroll
        for (int n = 0; n < E / 16; ++n) {
            const uint4 x = columns<D>(tdo, 0, n, lane), y = columns<D>(tq, 0, n, lane);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                dv[n][j] = mma<T>(x, p[j], dv[n][j]);
                dk[n][j] = mma<T>(y, ds[j], dk[n][j]);
                dk[n][j] = mma<T>(y, lo[j], dk[n][j]);
            }
        }
        if (D == 128) reads_ahead<4, 6, E / 16>();
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = wk0 + 16 * j + col;
        if (row >= sk.count) continue;
        const int64_t t = sk.first + row;
        const float back = a.scale * (L::kMoves ? L::kBack * moving[j].back() : L::kBack);
        if (a.by_key.parts == 1) {
            uint16_t *to_k = a.dk.p + t * a.dk.token + kv * a.dk.head, *to_v = a.dv.p + t * a.dv.token + kv * a.dv.head;
#pragma unroll
            for (int n = 0; n < E / 16; ++n)
                if (16 * n < a.d) {
                    const f32x4 x = dk[n][j] * back, y = dv[n][j] * L::kBack;
                    *reinterpret_cast<uint2 *>(to_k + 16 * n + 4 * g) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
                    *reinterpret_cast<uint2 *>(to_v + 16 * n + 4 * g) = make_uint2(pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]));
                }
        } else {
            float *to = a.by_key.sums + ((part * (int64_t)a.tokens_k + t) * hkv + kv) * 2 * a.d;
#pragma unroll
            for (int n = 0; n < E / 16; ++n)
                if (16 * n < a.d) {
                    *reinterpret_cast<f32x4 *>(to + 16 * n + 4 * g) = dk[n][j] * back;
                    *reinterpret_cast<f32x4 *>(to + a.d + 16 * n + 4 * g) = dv[n][j] * L::kBack;
                }
        }
    }
}

// dK and dV from the sums of the parts
template <typename T>
__global__ __launch_bounds__(256) void attn_dkv_join_kernel(const Problem a)
{
    const int hkv = a.hq / a.group, quads = a.d >> 1;   // of a row of dK and one of dV
    Joined j;
    if (!join_rows(a.cu_k, a.sequences, a.tokens_k, hkv, j)) return;
    const int64_t step = (int64_t)a.tokens_k * hkv * 2 * a.d;
    for (int item = threadIdx.x; item < j.rows * quads; item += 256) {
        const int row = item / quads, i = 4 * (item - row * quads);
        const int64_t t = j.first + row;
        const float *from = a.by_key.sums + (t * hkv + j.head) * 2 * a.d + i;
        f32x4 x = *reinterpret_cast<const f32x4 *>(from);
        for (int p = 1; p < a.by_key.parts; ++p) x += *reinterpret_cast<const f32x4 *>(from + p * step);
        uint16_t *to = i < a.d ? a.dk.p + t * a.dk.token + j.head * a.dk.head + i : a.dv.p + t * a.dv.token + j.head * a.dv.head + i - a.d;
        *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    }
}

// dQ, over the keys that a workgroup's queries see, 32 at a time and wave: four waves of 32 queries (KS = 1), or two pairs, of which each wave takes half of a
// tile's keys (KS = 2): twice the workgroups, each of half the length, for twice the copies.  STATS: it reads the row statistics; else it forms them, and leaves them to dK and dV.
// lk, lv: two tiles of LDS each, for keys and values
template <typename T, int D, int E, int KS, bool STATS> __device__ __forceinline__ void dq_tile(const Problem &a, unsigned block, lds_byte *lk, lds_byte *lv)
{
    using L = Lift<T>;
    constexpr int BQ = 128 / KS, BK = 32 * KS, TILE = BK * 2 * D;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4, qw = KS == 2 ? wave & 1 : wave, first_key = KS == 2 ? 32 * (wave >> 1) : 0;
    const Unit unit = unit_of(block, a.hq / a.group, a.by_query.parts);
    const int kv = unit.head;
    int sequence, index;
    if (!find_queries(a, BQ, unit.tile, lane, sequence, index)) return;
    Queries s_;
    s_.init(span(a.cu_q, sequence, a.tokens_q), span(a.cu_k, sequence, a.tokens_k), a.group, a.causal, index, BQ, 32 * qw);
    const Span sk = s_.k;
    const int all_tiles = s_.seen > 0 ? (s_.seen + BK - 1) / BK : 0;
    const int begin = (int)((int64_t)all_tiles * unit.part / a.by_query.parts), tiles = (int)((int64_t)all_tiles * (unit.part + 1) / a.by_query.parts);
    uint4 q[2][E / 32], dO[2][E / 32];
    float lse[2], delta[2];   // (delta times what dS is taken by)
    Moving moving[2];
    int last[2];   // that a row sees
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int of_tile = 32 * qw + 16 * j + col;
        const bool live = s_.row0 + of_tile < s_.rows;
        const Queries::Row of = s_.row(a.group, kv, of_tile);
        const int64_t t = of.token;
        const int head = of.head;
        const int64_t at = (int64_t)head * a.tokens_q + t;
        last[j] = !live ? -1 : a.causal ? min(sk.count - 1, of.at + s_.ahead) : sk.count - 1;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < E / 32; ++k) {
            const int i = 32 * k + 8 * g;
            q[j][k] = i < a.d ? *reinterpret_cast<const uint4 *>(a.q.p + t * a.q.token + head * a.q.head + i) : make_uint4(0, 0, 0, 0);
            dO[j][k] = i < a.d ? *reinterpret_cast<const uint4 *>(a.dO.p + t * a.dO.token + head * a.dO.head + i) : make_uint4(0, 0, 0, 0);
            if (STATS) continue;
            if (i < a.d)
                sum += dot<T>(*reinterpret_cast<const uint4 *>(a.o.p + t * a.o.token + head * a.o.head + i),
                              a.rest != nullptr ? *reinterpret_cast<const uint2 *>(a.rest + (t * a.hq + head) * a.d + i) : make_uint2(0, 0), dO[j][k]);
        }
        if (STATS) {
            const float2 of_row = a.stats[at];
            lse[j] = of_row.x, delta[j] = of_row.y;
        } else {
            lse[j] = fmaf(a.lse[at], kLog2e, -L::kUp), delta[j] = column_sum(sum);
            if (g == 0 && wave < 4 / KS && unit.part == 0 && live) a.stats[at] = make_float2(lse[j], delta[j]);
        }
        if (L::kMoves) delta[j] *= moving[j].by;
    }
    const float c = a.scale * kLog2e;
    f32x4 dq[E / 16][2];
#pragma unroll
    for (int n = 0; n < E / 16; ++n) dq[n][0] = dq[n][1] = f32x4{};

    const uint16_t *keys = a.k.p + sk.first * a.k.token + kv * a.k.head, *values = a.v.p + sk.first * a.v.token + kv * a.v.head;
    Copy<D, BK, 4> ck, cv;
    ck.init(wave, lane, (int)a.k.token * 2, a.d), cv.init(wave, lane, (int)a.v.token * 2, a.d);
    auto copy = [&](int t) {
        const int left = sk.count - t * BK;
        if (left < BK) ck.offsets(left), cv.offsets(left);
        ck.start(keys + (int64_t)t * BK * a.k.token, lk + (t & 1) * TILE);
        cv.start(values + (int64_t)t * BK * a.v.token, lv + (t & 1) * TILE);
    };
    if (begin < tiles) copy(begin);
    for (int t = begin; t < tiles; ++t) {
        wait_and_barrier<0>();
        if (t + 1 < tiles) copy(t + 1);
        const int k0 = t * BK + first_key;
        if (k0 >= s_.wave_seen) continue;
        const lds_byte *tk = lk + (t & 1) * TILE, *tv = lv + (t & 1) * TILE;
        f32x4 s[2][2], dp[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = dp[i][0] = dp[i][1] = f32x4{};
#pragma unroll
        for (int k = 0; k < E / 32; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 x = rows<D>(tk, first_key + 16 * i, k, lane), y = rows<D>(tv, first_key + 16 * i, k, lane);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[i][j] = mma<T>(x, q[j][k], s[i][j]);
                    dp[i][j] = mma<T>(y, dO[j][k], dp[i][j]);
                }
            }
        uint4 ds[2], lo[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c, -lse[j])) * (L::kMoves ? fmaf(dp[i][j][r], moving[j].by, -delta[j]) : dp[i][j][r] - delta[j]);
            if (k0 + 32 > s_.wave_all) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[i][j][r] = k0 + 16 * i + 4 * g + r <= last[j] ? s[i][j][r] : 0.0f;
            }
        }
        if constexpr (L::kMoves) {
            float most[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) most[j] = largest(largest(0.0f, s[0][j]), s[1][j]);
            if (__any(most[0] >= 0x1p15f || most[1] >= 0x1p15f)) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float f = moving[j].step(most[j]);
                    delta[j] *= f, s[0][j] *= f, s[1][j] *= f;
#pragma unroll
                    for (int n = 0; n < E / 16; ++n) dq[n][j] *= f;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) ds[j] = operand<T>(s[0][j], s[1][j]), lo[j] = rest<T>(ds[j], s[0][j], s[1][j]);
#pragma unroll
        for (int n = 0; n < E / 16; ++n) {
            const uint4 x = columns<D>(tk, first_key, n, lane);
            dq[n][0] = mma<T>(x, ds[0], dq[n][0]);
            dq[n][1] = mma<T>(x, ds[1], dq[n][1]);
            dq[n][0] = mma<T>(x, lo[0], dq[n][0]);
            dq[n][1] = mma<T>(x, lo[1], dq[n][1]);
        }
    }
    if constexpr (L::kMoves) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < E / 16; ++n) dq[n][j] *= moving[j].back();
    }
    if constexpr (KS == 2) {   // the wave of a pair that has the later keys hands its sums over, in LDS that no wave reads any more
        constexpr int SUMS = E / 16 * 2 * 1024;
        static_assert(SUMS <= 2 * TILE, "the sums must fit");
        lds_byte *const to = qw == 0 ? lk : lv;
        wait_and_barrier<0>();
        if (wave >= 2) {
#pragma unroll
            for (int n = 0; n < E / 16; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) lds_store(to + (2 * n + j) * 1024 + 16 * lane, dq[n][j]);
        }
        wait_and_barrier<0>();
        if (wave >= 2) return;
#pragma unroll
        for (int n = 0; n < E / 16; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) dq[n][j] += __builtin_bit_cast(f32x4, lds_load(to + (2 * n + j) * 1024 + 16 * lane));
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = 32 * qw + 16 * j + col;
        if (s_.row0 + row >= s_.rows) continue;
        const Queries::Row of = s_.row(a.group, kv, row);
        const int64_t token = of.token;
        const int head = of.head;
#pragma unroll
        for (int n = 0; n < E / 16; ++n)
            if (16 * n < a.d) {
                const f32x4 x = dq[n][j] * (a.scale * L::kBack);
                if (a.by_query.parts == 1)
                    *reinterpret_cast<uint2 *>(a.dq.p + token * a.dq.token + head * a.dq.head + 16 * n + 4 * g) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
                else
                    *reinterpret_cast<f32x4 *>(a.by_query.sums + ((unit.part * (int64_t)a.tokens_q + token) * a.hq + head) * a.d + 16 * n + 4 * g) = x;
            }
    }
}

// Large grids: dQ, which runs first and leaves the row statistics; dK and dV
template <typename T, int D, int E>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(const Problem a)
{
    constexpr int TILE = 32 * 2 * D;
    __shared__ __align__(16) unsigned char lds_k[2 * TILE], lds_v[2 * TILE];
    dq_tile<T, D, E, 1, false>(a, blockIdx.x, (lds_byte *)lds_k, (lds_byte *)lds_v);
}
template <typename T, int D, int E>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attn_dkv_kernel(const Problem a)
{
    using C = Backward<D>;
    __shared__ __align__(16) unsigned char values[C::VALUES], stages[2 * C::STAGE];
    dkv_tile<T, D, E>(a, blockIdx.x, (lds_byte *)values, (lds_byte *)stages);
}
// Small grids: all three in one launch, since neither fills the device to its end; the row statistics are formed before.  (The gradients, in turn and so: 16 heads
// of 128, 2048 tokens 193 and 119 us; 12 heads of 64, 1024 tokens 70 and 38, 8 x 1024 tokens 106 and 94.  At four workgroups a
// compute unit, 32 heads on 8 of 128 and 4096 tokens, 620 both ways.)
template <typename T, int D, int E>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attn_bwd_kernel(const Problem a)
{
    using C = Backward<D>;
    static_assert(2 * 64 * 2 * D <= C::VALUES && 2 * 64 * 2 * D <= 2 * C::STAGE, "two tiles must fit");
    __shared__ __align__(16) unsigned char values[C::VALUES], stages[2 * C::STAGE];
    if (blockIdx.x < a.key_blocks) dkv_tile<T, D, E>(a, blockIdx.x, (lds_byte *)values, (lds_byte *)stages);
    else dq_tile<T, D, E, 2, true>(a, blockIdx.x - a.key_blocks, (lds_byte *)values, (lds_byte *)stages);
}
// stats[h][t]: what a row's exponents are taken from, and delta = dO.O; by LANES lanes, one for each of a row's pieces of 16 bytes, for four rows at a time so that
// enough loads are under way.  (Both passes of 8 x 1024 tokens of 12 heads of 64: 108.9 us with one row, 107.6 with four.)
constexpr int kStatsRows = 4;
template <typename T, int LANES>
__global__ __launch_bounds__(256) void attn_stats_kernel(const Problem a)
{
    using L = Lift<T>;
    constexpr int ROWS = 256 / LANES;   // of a workgroup at a time
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t rows = (int64_t)a.tokens_q * a.hq, first = (int64_t)blockIdx.x * (ROWS * kStatsRows) + threadIdx.x / LANES;
    uint4 x[kStatsRows], y[kStatsRows];   // of dO, of O
    uint2 left[kStatsRows];
    float lse[kStatsRows];
    int64_t at[kStatsRows];
#pragma unroll
    for (int r = 0; r < kStatsRows; ++r) {
        const int64_t item = min(first + r * ROWS, rows - 1), t = item / a.hq;
        const int h = (int)(item - t * a.hq), i = min(8 * lane, a.d - 8);
        x[r] = *reinterpret_cast<const uint4 *>(a.dO.p + t * a.dO.token + h * a.dO.head + i);
        y[r] = *reinterpret_cast<const uint4 *>(a.o.p + t * a.o.token + h * a.o.head + i);
        left[r] = a.rest != nullptr ? *reinterpret_cast<const uint2 *>(a.rest + item * a.d + i) : make_uint2(0, 0);
        at[r] = h * (int64_t)a.tokens_q + t, lse[r] = a.lse[at[r]];
    }
#pragma unroll
    for (int r = 0; r < kStatsRows; ++r) {
        float sum = 8 * lane < a.d ? dot<T>(y[r], left[r], x[r]) : 0.0f;
#pragma unroll
        for (int s = 1; s < LANES; s <<= 1) sum += __shfl_xor(sum, s);
        if (lane == 0 && first + r * ROWS < rows) a.stats[at[r]] = make_float2(fmaf(lse[r], kLog2e, -L::kUp), sum);
    }
}

// dQ from the sums of the parts
template <typename T>
__global__ __launch_bounds__(256) void attn_dq_join_kernel(const Problem a)
{
    Joined j;
    if (!join_rows(a.cu_q, a.sequences, a.tokens_q, a.hq, j)) return;
    const int quads = a.d >> 2;
    const int64_t step = (int64_t)a.tokens_q * a.hq * a.d;
    for (int item = threadIdx.x; item < j.rows * quads; item += 256) {
        const int row = item / quads, i = 4 * (item - row * quads);
        const int64_t t = j.first + row;
        const float *from = a.by_query.sums + (t * a.hq + j.head) * a.d + i;
        f32x4 x = *reinterpret_cast<const f32x4 *>(from);
        for (int p = 1; p < a.by_query.parts; ++p) x += *reinterpret_cast<const f32x4 *>(from + p * step);
        *reinterpret_cast<uint2 *>(a.dq.p + t * a.dq.token + j.head * a.dq.head + i) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    }
}

// ------------------------------------------------------------------ host
static int check_shape(const s24_attn_shape *s, s24_dtype dt)
{
    S24_REQUIRE(s != nullptr && s->cu_q != nullptr && s->cu_k != nullptr, S24_ERR_NULL);
    S24_REQUIRE(s24_valid_dtype(dt), S24_ERR_DTYPE);
    S24_REQUIRE(s->sequences >= 0 && s->tokens_q >= 0 && s->tokens_k >= 0 && s->hq > 0 && s->hkv > 0 && s->hq % s->hkv == 0, S24_ERR_SHAPE);
    S24_REQUIRE(s->sequences < INT32_MAX / 2 && s->tokens_q < INT32_MAX / 2 && s->tokens_k < INT32_MAX / 2 && s->hq < 65536, S24_ERR_SHAPE);
    S24_REQUIRE((s->tokens_q > s->tokens_k ? s->tokens_q : s->tokens_k) * (s->hq / s->hkv) < INT32_MAX / 2, S24_ERR_SHAPE);
    S24_REQUIRE(s->d >= 16 && s->d % 16 == 0, S24_ERR_SHAPE);
    S24_REQUIRE(s->scale > 0.0f && s->scale <= 3.0e38f, S24_ERR_SHAPE);
    S24_REQUIRE(s24_aligned(s->cu_q, 4) && s24_aligned(s->cu_k, 4) && s24_aligned(s->o_rest, 16), S24_ERR_ALIGN);
    S24_REQUIRE(dt != S24_F32 && s->d <= 128, S24_ERR_UNSUPPORTED);
    return S24_OK;
}
// Workgroups (of one part) that go over the keys, for tiles of `rows` rows: the queries of a group of heads
static int64_t query_groups(const s24_attn_shape *s, int rows)
{
    return (s->tokens_q * (s->hq / s->hkv) / rows + (s->tokens_q < s->sequences ? s->tokens_q : s->sequences)) * s->hkv;
}
static Rows rows_of(const s24_heads *v) { return {static_cast<const uint16_t *>(v->data), v->token, v->head}; }
static Out out_of(const s24_heads *v) { return {static_cast<uint16_t *>(v->data), v->token, v->head}; }
static Problem problem_of(const s24_attn_shape *s)
{
    Problem a{};
    a.cu_q = s->cu_q, a.cu_k = s->cu_k, a.rest = s->o_rest;
    a.sequences = (int)s->sequences, a.tokens_q = (int)s->tokens_q, a.tokens_k = (int)s->tokens_k;
    a.hq = (int)s->hq, a.group = (int)(s->hq / s->hkv), a.d = (int)s->d, a.causal = s->causal != 0, a.scale = s->scale;
    // By length, unless the launch has many times the workgroups that the device holds, and the order matters less than keys that are still in the L2s; or the
    // queries are few for their keys, and a sequence's tiles are of nearly one length.  (Sequence by sequence and by length, forward: 8 x 2048 tokens of 8 heads of
    // 128 115 and 83 us, 6 x 1536 of 16 heads 91 and 80, 16 x 1024 of 32 heads on 8 227 and 236, 4 x 4096 of 32 heads 549 and 587; 1000 tokens after 18000, of 64
    // heads on 8, 308 and 328.  Tiles of keys gain at all sizes: gradients of 16 x 1024 tokens 866 and 712 us, of 8 x 2048 442 and 328.)
    a.mix_queries = s->sequences > 1 && s->tokens_k <= 2 * s->tokens_q && query_groups(s, 128) <= 8 * (int64_t)s24_cu_count();
    a.mix_keys = s->sequences > 1;
    return a;
}
}  // namespace s24_attn

using namespace s24_attn;

namespace s24_attn {
// Of a long one among the sequences, whose lengths the host does not know: of several, twice the average
static double per_sequence(int64_t tokens, const s24_attn_shape *s) { return (double)tokens * (s->sequences > 1 ? 2.0 / (double)s->sequences : 1.0); }
static double busy_keys(const s24_attn_shape *s)   // part of the keys that a query sees
{
    return s->causal && s->tokens_k > 0 ? 1.0 - 0.5 * (s->tokens_q < s->tokens_k ? (double)s->tokens_q / (double)s->tokens_k : 1.0) : 1.0;
}
static int forward_parts(const s24_attn_shape *s)
{
    return parts_for((double)query_groups(s, 128), per_sequence(s->tokens_k, s) / 64.0, busy_keys(s), s->d <= 64 ? 1.05 : 1.5,
                     (double)s->tokens_q * (double)s->hq * (double)s->d * 4.0);
}
// Backward.  joint: below four workgroups of 128 queries a compute unit all three gradients come from one launch, dQ from tiles of 64 queries (attn_bwd_kernel).
struct Plan { bool joint; int query_parts, key_parts; };
static Plan plan_backward(const s24_attn_shape *s)
{
    Plan p{query_groups(s, 128) < 4 * (int64_t)s24_cu_count(), 1, 1};
    if (p.joint)
        p.query_parts = parts_for((double)query_groups(s, 64), per_sequence(s->tokens_k, s) / 64.0, busy_keys(s), s->d <= 64 ? 0.66 : 1.1,
                                  (double)s->tokens_q * (double)s->hq * (double)s->d * 4.0);
    p.key_parts = parts_for((double)(most_tiles(s->tokens_k, s->sequences, 128) * s->hkv), per_sequence(s->tokens_q, s) / 32.0 * (double)(s->hq / s->hkv), s->causal ? 0.5 : 1.0,
                            s->d <= 64 ? 1.0 : 1.3, (double)s->tokens_k * (double)s->hkv * (double)s->d * 8.0);
    return p;
}
static bool sane(const s24_attn_shape *s)
{
    return s != nullptr && s->tokens_q >= 0 && s->tokens_k >= 0 && s->sequences >= 0 && s->hq > 0 && s->hkv > 0 && s->hq % s->hkv == 0 && s->d > 0;
}
static int64_t stats_bytes(const s24_attn_shape *s) { return (s->tokens_q * s->hq * (int64_t)sizeof(float2) + 15) / 16 * 16; }

template <typename T> static int forward(const Problem &a, dim3 grid, dim3 join, hipStream_t st)
{
    const dim3 block(256);
    if (a.d <= 64) attn_fwd_kernel<T, 64, 64><<<grid, block, 0, st>>>(a);
    else if (a.d <= 96) attn_fwd_kernel<T, 128, 96><<<grid, block, 0, st>>>(a);
    else attn_fwd_kernel<T, 128, 128><<<grid, block, 0, st>>>(a);
    if (a.by_query.parts > 1) attn_fwd_join_kernel<T><<<join, block, 0, st>>>(a);
    return s24_launch_status();
}
}  // namespace s24_attn

extern "C" int64_t s24_attn_fwd_workspace(const s24_attn_shape *shape)
{
    if (!sane(shape)) return 0;
    const int64_t parts = forward_parts(shape);
    return parts > 1 ? parts * (stats_bytes(shape) + shape->tokens_q * shape->hq * shape->d * 4) : 0;
}

extern "C" int s24_attn_fwd(const s24_attn_shape *shape, const s24_heads *Q, const s24_heads *K, const s24_heads *V, const s24_heads *O, float *lse,
                            void *workspace, int64_t workspace_bytes, s24_dtype dt, void *stream)
{
    S24_TRY(check_shape(shape, dt));
    S24_TRY(check_rows(Q, shape->tokens_q, shape->hq, shape->d, false));
    S24_TRY(check_rows(K, shape->tokens_k, shape->hkv, shape->d, false));
    S24_TRY(check_rows(V, shape->tokens_k, shape->hkv, shape->d, false));
    S24_TRY(check_rows(O, shape->tokens_q, shape->hq, shape->d, true));
    const int64_t need = s24_attn_fwd_workspace(shape);
    S24_REQUIRE(workspace != nullptr || need == 0, S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(lse, 4) && s24_aligned(workspace, 16), S24_ERR_ALIGN);
    S24_REQUIRE(workspace_bytes >= need, S24_ERR_SHAPE);
    const int parts = forward_parts(shape);
    const int64_t groups = query_groups(shape, 128) * parts;
    const int64_t join = most_tiles(shape->tokens_q, shape->sequences, kJoinRows) * shape->hq;
    S24_REQUIRE(groups <= kMostGroups && (parts == 1 || join <= kMostGroups), S24_ERR_SHAPE);
    if (groups == 0) return S24_OK;
    Problem a = problem_of(shape);
    a.q = rows_of(Q), a.k = rows_of(K), a.v = rows_of(V), a.out = out_of(O), a.lse = lse;
    a.weights = static_cast<float2 *>(workspace);
    a.by_query = {parts, reinterpret_cast<float *>(static_cast<char *>(workspace) + parts * stats_bytes(shape))};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups), join_grid((unsigned)join);
    return dt == S24_BF16 ? forward<uint16_t>(a, grid, join_grid, st) : forward<s24_half>(a, grid, join_grid, st);
}

namespace s24_attn {
template <typename T, int D, int E> static int backward(Problem a, bool joint, int64_t query_groups, hipStream_t st)
{
    const dim3 block(256);
    const int64_t hkv = a.hq / a.group, key_groups = most_tiles(a.tokens_k, a.sequences, 128) * hkv * a.by_key.parts;
    if (query_groups == 0 && key_groups == 0) return S24_OK;
    const bool together = joint && query_groups > 0;
    const int64_t rows = (int64_t)a.tokens_q * a.hq, of_group = 2048 / D * kStatsRows, stats = (rows + of_group - 1) / of_group, key_blocks = (key_groups + 7) / 8 * 8;
    const int64_t dq_join = a.by_query.parts > 1 ? most_tiles(a.tokens_q, a.sequences, kJoinRows) * a.hq : 0, dkv_join = a.by_key.parts > 1 ? most_tiles(a.tokens_k, a.sequences, kJoinRows) * hkv : 0;
    S24_REQUIRE((together ? key_blocks + query_groups <= kMostGroups && stats <= kMostGroups : query_groups <= kMostGroups && key_groups <= kMostGroups) && dq_join <= kMostGroups &&
                dkv_join <= kMostGroups, S24_ERR_SHAPE);
    if (together) {
        a.key_blocks = (unsigned)key_blocks;   // dQ's workgroups meet the XCDs as they would in a launch of their own
        attn_stats_kernel<T, D / 8><<<dim3((unsigned)stats), block, 0, st>>>(a);
        attn_bwd_kernel<T, D, E><<<dim3(a.key_blocks + (unsigned)query_groups), block, 0, st>>>(a);
    } else {
        if (query_groups > 0) attn_dq_kernel<T, D, E><<<dim3((unsigned)query_groups), block, 0, st>>>(a);
        if (key_groups > 0) attn_dkv_kernel<T, D, E><<<dim3((unsigned)key_groups), block, 0, st>>>(a);
    }
    if (query_groups > 0 && dq_join > 0) attn_dq_join_kernel<T><<<dim3((unsigned)dq_join), block, 0, st>>>(a);
    if (key_groups > 0 && dkv_join > 0) attn_dkv_join_kernel<T><<<dim3((unsigned)dkv_join), block, 0, st>>>(a);
    return s24_launch_status();
}
template <typename T> static int backward(const Problem &a, bool joint, int64_t query_groups, hipStream_t st)
{
    return a.d <= 64 ? backward<T, 64, 64>(a, joint, query_groups, st) : a.d <= 96 ? backward<T, 128, 96>(a, joint, query_groups, st) : backward<T, 128, 128>(a, joint, query_groups, st);
}
static int64_t query_sums(const s24_attn_shape *s, int parts) { return parts > 1 ? parts * s->tokens_q * s->hq * s->d * 4 : 0; }
static int64_t key_sums(const s24_attn_shape *s, int parts) { return parts > 1 ? parts * s->tokens_k * s->hkv * s->d * 8 : 0; }
}  // namespace s24_attn

extern "C" int64_t s24_attn_bwd_workspace(const s24_attn_shape *shape)
{
    if (!sane(shape)) return 0;
    const Plan plan = plan_backward(shape);
    return stats_bytes(shape) + query_sums(shape, plan.query_parts) + key_sums(shape, plan.key_parts);
}

extern "C" int s24_attn_bwd(const s24_attn_shape *shape, const s24_heads *Q, const s24_heads *K, const s24_heads *V, const s24_heads *O,
                            const s24_heads *dO, const float *lse, const s24_heads *dQ, const s24_heads *dK, const s24_heads *dV, void *workspace,
                            int64_t workspace_bytes, s24_dtype dt, void *stream)
{
    S24_TRY(check_shape(shape, dt));
    for (const s24_heads *x : {Q, O, dO, dQ}) S24_TRY(check_rows(x, shape->tokens_q, shape->hq, shape->d, x == dQ));
    for (const s24_heads *x : {K, V, dK, dV}) S24_TRY(check_rows(x, shape->tokens_k, shape->hkv, shape->d, x == dK || x == dV));
    S24_REQUIRE((lse != nullptr && workspace != nullptr) || shape->tokens_q == 0, S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(lse, 4) && s24_aligned(workspace, 16), S24_ERR_ALIGN);
    S24_REQUIRE(workspace_bytes >= s24_attn_bwd_workspace(shape), S24_ERR_SHAPE);
    S24_REQUIRE(most_tiles(shape->tokens_q, shape->sequences, kJoinRows) * shape->hq <= INT32_MAX / 2 &&
                most_tiles(shape->tokens_k, shape->sequences, kJoinRows) * shape->hkv <= INT32_MAX / 2, S24_ERR_SHAPE);   // (tiles are numbered in an int)
    Problem a = problem_of(shape);
    a.q = rows_of(Q), a.k = rows_of(K), a.v = rows_of(V), a.o = rows_of(O), a.dO = rows_of(dO);
    a.dq = out_of(dQ), a.dk = out_of(dK), a.dv = out_of(dV);
    a.lse = const_cast<float *>(lse), a.stats = static_cast<float2 *>(workspace);
    const Plan plan = plan_backward(shape);
    char *const sums = static_cast<char *>(workspace) + stats_bytes(shape);
    a.by_query = {plan.query_parts, reinterpret_cast<float *>(sums)};
    a.by_key = {plan.key_parts, reinterpret_cast<float *>(sums + query_sums(shape, plan.query_parts))};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t groups = query_groups(shape, plan.joint ? 64 : 128) * plan.query_parts;
    return dt == S24_BF16 ? backward<uint16_t>(a, plan.joint, groups, st) : backward<s24_half>(a, plan.joint, groups, st);
}
