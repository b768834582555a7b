// Attention over packed sequences, forward and backward (the training step's other half, and the reading of prompts).
//
// S_ij = c q_i.k_j over the visible pairs, P = softmax of its rows, O = P V.  Forward: one pass over the keys with the running maximum and sum
// of each row; S^T is formed with the keys as rows, so that a lane holds one query's scores, the row statistics need no exchange between lanes
// but a rare one, and the rounded P is the second product's operand as it lies in the registers.
// Backward, from lse_i = log sum_j exp S_ij and delta_i = dO_i.O_i:  P_ij = exp(S_ij - lse_i),  dV = P^T dO,  dS_ij = P_ij (dO_i.v_j - delta_i),
// dQ = c dS K,  dK = c dS^T Q.
// Sums run over queries for dK and dV and over keys for dQ: two kernels, each of which forms S and dO V^T for itself (7 products instead
// of 5).  One kernel would have to add to dQ from many workgroups, in an order that no two runs share.
#include "s24_attn.h"

#include <math.h>

namespace s24_attn {

struct Rows { const uint16_t *p; int64_t token, head; };   // element (t, h, i) at p + t*token + h*head + i
struct Out { uint16_t *p; int64_t token, head; };
struct Problem {
    Rows q, k, v, o, dO;
    Out out, dq, dk, dv;
    float *lse;            // [hq][tokens_q]
    float2 *stats;         // [hq][tokens_q], of the backward pass: what a row's exponents are taken from, and delta
    float *sums;           // [parts][tokens_k][hkv][2 d]
    int parts;
    const int *cu_q, *cu_k;
    int sequences, tokens_q, tokens_k, hq, group, d, causal;
    float scale;
};

// ------------------------------------------------------------------ forward
// Four waves of 32 queries; keys and values in tiles of 64, two of them in LDS: the next one is copied during the work on this one.
template <int D> struct Forward {
    static constexpr int BQ = 128, BK = 64, TILE = BK * 2 * D;
};

// Scores whose maximum grew by less than this (as a power of two) keep the reference they have: P then reaches 2^8, which the 16-bit types hold with
// the same relative precision, and the sums stay far inside fp32.
constexpr float kGrowth = 8.0f;

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(const Problem a)
{
    using C = Forward<D>;
    __shared__ __align__(16) unsigned char lds_k[2][C::TILE], lds_v[2][C::TILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int tile = blockIdx.x / a.hq, head = head_of(blockIdx.x - tile * a.hq, a.hq), kv = head / a.group;
    int sequence, index, count;
    if (!find_tile(a.cu_q, a.sequences, a.tokens_q, C::BQ, tile, lane, sequence, index, count)) return;
    const Span sq = span(a.cu_q, sequence, a.tokens_q), sk = span(a.cu_k, sequence, a.tokens_k);
    const int q0 = (count - 1 - index) * C::BQ;    // the last ones see the most keys: they go first
    const int ahead = sk.count - sq.count;         // query i sees the keys up to i + ahead
    const int wq0 = q0 + 32 * wave;                // this wave's queries
    const int seen = a.causal ? min(sk.count, q0 + C::BQ + ahead) : sk.count;            // keys that some query of the tile may see
    const int wave_seen = a.causal ? min(sk.count, wq0 + 32 + ahead) : sk.count;         // of the wave
    const int wave_all = a.causal ? min(sk.count, wq0 + 1 + ahead) : sk.count;           // keys that all its queries see
    const int tiles = seen > 0 ? (seen + C::BK - 1) / C::BK : 0;

    uint4 q[2][D / 32];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint16_t *row = a.q.p + (int64_t)(sq.first + min(wq0 + 16 * j + col, sq.count - 1)) * a.q.token + head * a.q.head;
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
            q[j][k] = 32 * k + 8 * g < a.d ? *reinterpret_cast<const uint4 *>(row + 32 * k + 8 * g) : make_uint4(0, 0, 0, 0);
    }
    const float c = a.scale * kLog2e;
    float m[2] = {-1e30f, -1e30f}, l[2] = {0.0f, 0.0f};
    f32x4 o[D / 16][2];
#pragma unroll
    for (int n = 0; n < D / 16; ++n) o[n][0] = o[n][1] = f32x4{};

    const uint16_t *keys = a.k.p + sk.first * a.k.token + kv * a.k.head, *values = a.v.p + sk.first * a.v.token + kv * a.v.head;
    Copy<D, C::BK, 4> ck, cv;
    ck.init(wave, lane, (int)a.k.token * 2, a.d), cv.init(wave, lane, (int)a.v.token * 2, a.d);
    auto copy = [&](int t) {
        const int left = sk.count - t * C::BK;
        if (left < C::BK) ck.offsets(left), cv.offsets(left);
        ck.start(keys + (int64_t)t * C::BK * a.k.token, (lds_byte *)lds_k[t & 1]);
        cv.start(values + (int64_t)t * C::BK * a.v.token, (lds_byte *)lds_v[t & 1]);
    };
    if (tiles > 0) copy(0);
    for (int t = 0; t < tiles; ++t) {
        wait_and_barrier<0>();
        if (t + 1 < tiles) copy(t + 1);
        const int k0 = t * C::BK;
        if (k0 >= wave_seen) continue;
        const lds_byte *tk = (const lds_byte *)lds_k[t & 1], *tv = (const lds_byte *)lds_v[t & 1];
        f32x4 s[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = f32x4{};
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 f = rows<D>(tk, 16 * i, k, lane);
                s[i][0] = mma<T>(f, q[0][k], s[i][0]);
                s[i][1] = mma<T>(f, q[1][k], s[i][1]);
            }
        if (k0 + C::BK > wave_all) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int last = a.causal ? min(sk.count - 1, wq0 + 16 * j + col + ahead) : sk.count - 1;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[i][j][r] = k0 + 16 * i + 4 * g + r <= last ? s[i][j][r] : -INFINITY;
            }
        }
        float top[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            top[j] = s[0][j][0];
#pragma unroll
            for (int i = 0; i < 4; ++i)
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
                for (int n = 0; n < D / 16; ++n) o[n][j] *= shrink;
            }
        }
        uint4 p[2][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c, -m[j]));
                    l[j] += s[i][j][r];
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) p[u][j] = operand<T>(s[2 * u][j], s[2 * u + 1][j]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                const uint4 f = columns<D>(tv, 32 * u, n, lane);
                o[n][0] = mma<T>(f, p[u][0], o[n][0]);
                o[n][1] = mma<T>(f, p[u][1], o[n][1]);
            }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = wq0 + 16 * j + col;
        const float sum = column_sum(l[j]), inverse = sum > 0.0f ? 1.0f / sum : 0.0f;
        if (row >= sq.count) continue;
        uint16_t *out = a.out.p + (int64_t)(sq.first + row) * a.out.token + head * a.out.head;
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
            if (16 * n < a.d)
                *reinterpret_cast<uint2 *>(out + 16 * n + 4 * g) =
                    make_uint2(pack2<T>(o[n][j][0] * inverse, o[n][j][1] * inverse), pack2<T>(o[n][j][2] * inverse, o[n][j][3] * inverse));
        if (a.lse != nullptr && g == 0)
            a.lse[(int64_t)head * a.tokens_q + sq.first + row] = sum > 0.0f ? (m[j] + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
    }
}

// ------------------------------------------------------------------ backward
// P is formed times 2^kUp, from lse - kUp: exp2 gives zero for what fp32 has no normal number for, and binary16 holds weights below 2^-14 with fewer bits.
// In bf16 the factor goes through dS to the end of the sums; binary16 has no room for it there, so dP and delta take it back.
template <typename T> struct Lift;
template <> struct Lift<uint16_t> { static constexpr float kUp = 32.0f, kDown = 1.0f, kOfP = 0x1p-32f, kOfDs = 0x1p-32f; };
template <> struct Lift<s24_half> { static constexpr float kUp = 15.0f, kDown = 0x1p-15f, kOfP = 0x1p-15f, kOfDs = 1.0f; };

// dK and dV of 128 keys of a key-value head, four waves of 32: over the query heads of the group and their queries, 32 at a time.
// S has the queries as rows, so that P and dS are, as they lie, the operands that contract over the queries.
template <int D> struct Backward {
    static constexpr int BK = 128, BQ = 32, TILE = BQ * 2 * D, STAGE = 2 * TILE + 8 * BQ, VALUES = BK * 2 * D;   // a stage: queries, gradients, row statistics
};
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attn_dkv_kernel(const Problem a)
{
    using C = Backward<D>;
    using L = Lift<T>;
    __shared__ __align__(16) unsigned char stages[2][C::STAGE], values[C::VALUES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int hkv = a.hq / a.group;
    const int units = hkv * a.parts, tile = blockIdx.x / units, unit = head_of(blockIdx.x - tile * units, units), kv = unit / a.parts, part = unit - kv * a.parts;
    int sequence, index, count;
    if (!find_tile(a.cu_k, a.sequences, a.tokens_k, C::BK, tile, lane, sequence, index, count)) return;
    const Span sq = span(a.cu_q, sequence, a.tokens_q), sk = span(a.cu_k, sequence, a.tokens_k);
    const int k0 = index * C::BK, wk0 = k0 + 32 * wave;   // the first keys are seen by the most queries: they go first
    const int ahead = sk.count - sq.count;
    const int first = a.causal ? max(0, k0 - ahead) / C::BQ : 0;                // query tiles
    const int each = max(0, (sq.count + C::BQ - 1) / C::BQ - first);
    // the steps of all heads of the group, and of them this part's
    const int64_t all_steps = (int64_t)each * a.group;
    const int begin = (int)(all_steps * part / a.parts), steps = (int)(all_steps * (part + 1) / a.parts) - begin;

    // The keys' fragments stay in registers, the values' come from LDS: with both, two waves would not fit a SIMD (3.6 ms instead of MEASURE for 8192 tokens,
    // 64 heads on 8 of 128).
    uint4 fk[2][D / 32];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t t = sk.first + min(wk0 + 16 * j + col, sk.count - 1);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const int i = 32 * k + 8 * g;
            fk[j][k] = i < a.d ? *reinterpret_cast<const uint4 *>(a.k.p + t * a.k.token + kv * a.k.head + i) : make_uint4(0, 0, 0, 0);
        }
    }
    lds_byte *const tv = (lds_byte *)values;
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
    f32x4 dk[D / 16][2], dv[D / 16][2];
#pragma unroll
    for (int n = 0; n < D / 16; ++n) dk[n][0] = dk[n][1] = dv[n][0] = dv[n][1] = f32x4{};
    const float c = a.scale * kLog2e;

    Copy<D, C::BQ, 4> cq, cdo;
    cq.init(wave, lane, (int)a.q.token * 2, a.d), cdo.init(wave, lane, (int)a.dO.token * 2, a.d);
    int next_head = kv * a.group + (each > 0 ? begin / each : 0), next_tile = first + (each > 0 ? begin % each : 0), buffer = 0;
    int qt = next_tile;
    auto copy = [&](int stage) {
        const int left = sq.count - next_tile * C::BQ;
        cq.offsets(min(left, C::BQ)), cdo.offsets(min(left, C::BQ));
        const int64_t t = sq.first + next_tile * C::BQ;
        lds_byte *to = (lds_byte *)stages[stage];
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
        if (a.causal && q0 + C::BQ - 1 + ahead < wk0) continue;   // no query of the tile sees a key of the wave
        const lds_byte *tq = (const lds_byte *)stages[now], *tdo = tq + C::TILE, *stats = tdo + C::TILE;
        f32x4 s[2][2], dp[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = dp[i][0] = dp[i][1] = f32x4{};
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
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
        f32x4 lse[2], delta[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float4 two = __builtin_bit_cast(float4, lds_load(stats + 8 * (16 * i + 4 * g + 2 * r)));
                lse[i][2 * r] = two.x, delta[i][2 * r] = two.y, lse[i][2 * r + 1] = two.z, delta[i][2 * r + 1] = two.w;
            }
        const bool all = q0 + C::BQ <= sq.count && wk0 + 32 <= sk.count && (!a.causal || wk0 + 31 <= q0 + ahead);
        uint4 p[2], ds[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c, -lse[i][r]));
                    dp[i][j][r] = s[i][j][r] * fmaf(dp[i][j][r], L::kDown, -delta[i][r]);
                }
            if (!all) {   // whatever stands in rows past the last, nothing of it stays
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
            p[j] = operand<T>(s[0][j], s[1][j]), ds[j] = operand<T>(dp[0][j], dp[1][j]);
        }
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            const uint4 x = columns<D>(tdo, 0, n, lane), y = columns<D>(tq, 0, n, lane);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                dv[n][j] = mma<T>(x, p[j], dv[n][j]);
                dk[n][j] = mma<T>(y, ds[j], dk[n][j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = wk0 + 16 * j + col;
        if (row >= sk.count) continue;
        const int64_t t = sk.first + row;
        if (a.parts == 1) {
            uint16_t *to_k = a.dk.p + t * a.dk.token + kv * a.dk.head, *to_v = a.dv.p + t * a.dv.token + kv * a.dv.head;
#pragma unroll
            for (int n = 0; n < D / 16; ++n)
                if (16 * n < a.d) {
                    const f32x4 x = dk[n][j] * (a.scale * L::kOfDs), y = dv[n][j] * L::kOfP;
                    *reinterpret_cast<uint2 *>(to_k + 16 * n + 4 * g) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
                    *reinterpret_cast<uint2 *>(to_v + 16 * n + 4 * g) = make_uint2(pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]));
                }
        } else {
            float *to = a.sums + ((part * (int64_t)a.tokens_k + t) * hkv + kv) * 2 * a.d;
#pragma unroll
            for (int n = 0; n < D / 16; ++n)
                if (16 * n < a.d) {
                    *reinterpret_cast<f32x4 *>(to + 16 * n + 4 * g) = dk[n][j] * (a.scale * L::kOfDs);
                    *reinterpret_cast<f32x4 *>(to + a.d + 16 * n + 4 * g) = dv[n][j] * L::kOfP;
                }
        }
    }
}

// dK and dV of a few keys from the sums of the parts
constexpr int kJoinRows = 16;
template <typename T>
__global__ __launch_bounds__(256) void attn_dkv_join_kernel(const Problem a)
{
    constexpr int BK = kJoinRows;
    const int hkv = a.hq / a.group, tile = blockIdx.x / hkv, kv = blockIdx.x - tile * hkv;
    int sequence, index, count;
    if (!find_tile(a.cu_k, a.sequences, a.tokens_k, BK, tile, threadIdx.x & 63, sequence, index, count)) return;
    const Span sk = span(a.cu_k, sequence, a.tokens_k);
    const int quads = a.d >> 1, n = min(BK, sk.count - index * BK) * quads;   // of a row of dK and one of dV
    const int64_t step = (int64_t)a.tokens_k * hkv * 2 * a.d;
    for (int item = threadIdx.x; item < n; item += 256) {
        const int row = item / quads, i = 4 * (item - row * quads);
        const int64_t t = sk.first + index * BK + row;
        const float *from = a.sums + (t * hkv + kv) * 2 * a.d + i;
        f32x4 x = *reinterpret_cast<const f32x4 *>(from);
        for (int p = 1; p < a.parts; ++p) x += *reinterpret_cast<const f32x4 *>(from + p * step);
        uint16_t *to = i < a.d ? a.dk.p + t * a.dk.token + kv * a.dk.head + i : a.dv.p + t * a.dv.token + kv * a.dv.head + i - a.d;
        *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    }
}

// dQ of 128 queries of a head, four waves of 32, over the keys they see, 32 at a time.  Runs first: it leaves the row statistics to dK and dV.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(const Problem a)
{
    using L = Lift<T>;
    constexpr int BQ = 128, BK = 32, TILE = BK * 2 * D;
    __shared__ __align__(16) unsigned char lds_k[2][TILE], lds_v[2][TILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int tile = blockIdx.x / a.hq, head = head_of(blockIdx.x - tile * a.hq, a.hq), kv = head / a.group;
    int sequence, index, count;
    if (!find_tile(a.cu_q, a.sequences, a.tokens_q, BQ, tile, lane, sequence, index, count)) return;
    const Span sq = span(a.cu_q, sequence, a.tokens_q), sk = span(a.cu_k, sequence, a.tokens_k);
    const int q0 = (count - 1 - index) * BQ, ahead = sk.count - sq.count, wq0 = q0 + 32 * wave;
    const int seen = a.causal ? min(sk.count, q0 + BQ + ahead) : sk.count;
    const int wave_seen = a.causal ? min(sk.count, wq0 + 32 + ahead) : sk.count;
    const int wave_all = wq0 + 32 > sq.count ? 0 : a.causal ? min(sk.count, wq0 + 1 + ahead) : sk.count;
    const int tiles = seen > 0 ? (seen + BK - 1) / BK : 0;
    uint4 q[2][D / 32], dO[2][D / 32];
    float lse[2], delta[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t t = sq.first + min(wq0 + 16 * j + col, sq.count - 1);
        const int64_t at = (int64_t)head * a.tokens_q + t;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const int i = 32 * k + 8 * g;
            q[j][k] = i < a.d ? *reinterpret_cast<const uint4 *>(a.q.p + t * a.q.token + head * a.q.head + i) : make_uint4(0, 0, 0, 0);
            dO[j][k] = i < a.d ? *reinterpret_cast<const uint4 *>(a.dO.p + t * a.dO.token + head * a.dO.head + i) : make_uint4(0, 0, 0, 0);
            const uint4 o = i < a.d ? *reinterpret_cast<const uint4 *>(a.o.p + t * a.o.token + head * a.o.head + i) : make_uint4(0, 0, 0, 0);
            using Num = s24_num<T>;
            const uint32_t xs[4] = {o.x, o.y, o.z, o.w}, ys[4] = {dO[j][k].x, dO[j][k].y, dO[j][k].z, dO[j][k].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf(Num::lo(xs[e]), Num::lo(ys[e]), fmaf(Num::hi(xs[e]), Num::hi(ys[e]), sum));
        }
        lse[j] = fmaf(a.lse[at], kLog2e, -L::kUp), delta[j] = column_sum(sum) * L::kDown;
        if (g == 0 && wq0 + 16 * j + col < sq.count) a.stats[at] = make_float2(lse[j], delta[j]);
    }
    const float c = a.scale * kLog2e;
    f32x4 dq[D / 16][2];
#pragma unroll
    for (int n = 0; n < D / 16; ++n) dq[n][0] = dq[n][1] = f32x4{};

    const uint16_t *keys = a.k.p + sk.first * a.k.token + kv * a.k.head, *values = a.v.p + sk.first * a.v.token + kv * a.v.head;
    Copy<D, BK, 4> ck, cv;
    ck.init(wave, lane, (int)a.k.token * 2, a.d), cv.init(wave, lane, (int)a.v.token * 2, a.d);
    auto copy = [&](int t) {
        const int left = sk.count - t * BK;
        if (left < BK) ck.offsets(left), cv.offsets(left);
        ck.start(keys + (int64_t)t * BK * a.k.token, (lds_byte *)lds_k[t & 1]);
        cv.start(values + (int64_t)t * BK * a.v.token, (lds_byte *)lds_v[t & 1]);
    };
    if (tiles > 0) copy(0);
    for (int t = 0; t < tiles; ++t) {
        wait_and_barrier<0>();
        if (t + 1 < tiles) copy(t + 1);
        const int k0 = t * BK;
        if (k0 >= wave_seen) continue;
        const lds_byte *tk = (const lds_byte *)lds_k[t & 1], *tv = (const lds_byte *)lds_v[t & 1];
        f32x4 s[2][2], dp[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = dp[i][0] = dp[i][1] = f32x4{};
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 x = rows<D>(tk, 16 * i, k, lane), y = rows<D>(tv, 16 * i, k, lane);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[i][j] = mma<T>(x, q[j][k], s[i][j]);
                    dp[i][j] = mma<T>(y, dO[j][k], dp[i][j]);
                }
            }
        uint4 ds[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int query = wq0 + 16 * j + col;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    s[i][j][r] = __builtin_amdgcn_exp2f(fmaf(s[i][j][r], c, -lse[j])) * fmaf(dp[i][j][r], L::kDown, -delta[j]);
            if (k0 + BK > wave_all) {
                const int last = query >= sq.count ? -1 : a.causal ? min(sk.count - 1, query + ahead) : sk.count - 1;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[i][j][r] = k0 + 16 * i + 4 * g + r <= last ? s[i][j][r] : 0.0f;
            }
            ds[j] = operand<T>(s[0][j], s[1][j]);
        }
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            const uint4 x = columns<D>(tk, 0, n, lane);
            dq[n][0] = mma<T>(x, ds[0], dq[n][0]);
            dq[n][1] = mma<T>(x, ds[1], dq[n][1]);
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = wq0 + 16 * j + col;
        if (row >= sq.count) continue;
        uint16_t *out = a.dq.p + (int64_t)(sq.first + row) * a.dq.token + head * a.dq.head;
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
            if (16 * n < a.d) {
                const f32x4 x = dq[n][j] * (a.scale * L::kOfDs);
                *reinterpret_cast<uint2 *>(out + 16 * n + 4 * g) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
            }
    }
}

// ------------------------------------------------------------------ host
static int check_shape(const s24_attn_shape *s, s24_dtype dt)
{
    S24_REQUIRE(s != nullptr && s->cu_q != nullptr && s->cu_k != nullptr, S24_ERR_NULL);
    S24_REQUIRE(s24_valid_dtype(dt), S24_ERR_DTYPE);
    S24_REQUIRE(s->sequences >= 0 && s->tokens_q >= 0 && s->tokens_k >= 0 && s->hq > 0 && s->hkv > 0 && s->hq % s->hkv == 0, S24_ERR_SHAPE);
    S24_REQUIRE(s->sequences < INT32_MAX / 2 && s->tokens_q < INT32_MAX / 2 && s->tokens_k < INT32_MAX / 2 && s->hq < 65536, S24_ERR_SHAPE);
    S24_REQUIRE(s->d >= 16 && s->d % 16 == 0, S24_ERR_SHAPE);
    S24_REQUIRE(s->scale > 0.0f && s->scale <= 3.0e38f, S24_ERR_SHAPE);
    S24_REQUIRE(s24_aligned(s->cu_q, 4) && s24_aligned(s->cu_k, 4), S24_ERR_ALIGN);
    S24_REQUIRE(dt != S24_F32 && s->d <= 128, S24_ERR_UNSUPPORTED);
    return S24_OK;
}
static Rows rows_of(const s24_heads *v) { return {static_cast<const uint16_t *>(v->data), v->token, v->head}; }
static Out out_of(const s24_heads *v) { return {static_cast<uint16_t *>(v->data), v->token, v->head}; }
static Problem problem_of(const s24_attn_shape *s)
{
    Problem a{};
    a.cu_q = s->cu_q, a.cu_k = s->cu_k;
    a.sequences = (int)s->sequences, a.tokens_q = (int)s->tokens_q, a.tokens_k = (int)s->tokens_k;
    a.hq = (int)s->hq, a.group = (int)(s->hq / s->hkv), a.d = (int)s->d, a.causal = s->causal != 0, a.scale = s->scale;
    return a;
}
}  // namespace s24_attn

using namespace s24_attn;

extern "C" int s24_attn_fwd(const s24_attn_shape *shape, const s24_heads *Q, const s24_heads *K, const s24_heads *V, const s24_heads *O, float *lse,
                            s24_dtype dt, void *stream)
{
    S24_TRY(check_shape(shape, dt));
    S24_TRY(check_rows(Q, shape->tokens_q, shape->hq, shape->d, false));
    S24_TRY(check_rows(K, shape->tokens_k, shape->hkv, shape->d, false));
    S24_TRY(check_rows(V, shape->tokens_k, shape->hkv, shape->d, false));
    S24_TRY(check_rows(O, shape->tokens_q, shape->hq, shape->d, true));
    S24_REQUIRE(s24_aligned(lse, 4), S24_ERR_ALIGN);
    const int64_t groups = most_tiles(shape->tokens_q, shape->sequences, Forward<128>::BQ) * shape->hq;
    S24_REQUIRE(groups <= kMostGroups, S24_ERR_SHAPE);
    if (groups == 0) return S24_OK;
    Problem a = problem_of(shape);
    a.q = rows_of(Q), a.k = rows_of(K), a.v = rows_of(V), a.out = out_of(O), a.lse = lse;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups), block(256);
    if (dt == S24_BF16) {
        if (a.d <= 64) attn_fwd_kernel<uint16_t, 64><<<grid, block, 0, st>>>(a);
        else attn_fwd_kernel<uint16_t, 128><<<grid, block, 0, st>>>(a);
    } else {
        if (a.d <= 64) attn_fwd_kernel<s24_half, 64><<<grid, block, 0, st>>>(a);
        else attn_fwd_kernel<s24_half, 128><<<grid, block, 0, st>>>(a);
    }
    return s24_launch_status();
}

namespace s24_attn {
// Parts in which the queries of a tile of keys are taken.  Two workgroups fit a compute unit, and when causal the first keys' have many times the work of
// the last ones': fewer than three for each unit are cut up into four or more.  (The sums of a part travel through memory in fp32: with 1.7 rounds, 12 heads of
// 64 and 8 x 1024 tokens, that costs more than it gives, 81 us to 67.)
static int64_t parts_of(const s24_attn_shape *s)
{
    const int64_t tiles = most_tiles(s->tokens_k, s->sequences, Backward<128>::BK) * s->hkv, units = s24_cu_count();
    if (tiles == 0 || tiles >= 3 * units) return 1;
    const int64_t parts = (4 * units + tiles - 1) / tiles, steps = (s->tokens_q / 32 + 1) * (s->hq / s->hkv);
    return parts > 8 ? 8 : parts > steps ? steps : parts;
}
static int64_t stats_bytes(const s24_attn_shape *s) { return (s->tokens_q * s->hq * (int64_t)sizeof(float2) + 15) / 16 * 16; }
}  // namespace s24_attn

extern "C" int64_t s24_attn_bwd_workspace(const s24_attn_shape *shape)
{
    if (shape == nullptr || shape->tokens_q < 0 || shape->tokens_k < 0 || shape->sequences < 0 || shape->hq <= 0 || shape->hkv <= 0 || shape->hq % shape->hkv != 0 || shape->d < 0) return 0;
    const int64_t parts = parts_of(shape);
    return stats_bytes(shape) + (parts > 1 ? parts * shape->tokens_k * shape->hkv * 2 * shape->d * 4 : 0);
}

namespace s24_attn {
template <typename T, int D> static int backward(const Problem &a, int64_t tiles_k, int64_t tiles_q, hipStream_t st)
{
    if (tiles_q > 0) attn_dq_kernel<T, D><<<dim3((unsigned)tiles_q), dim3(256), 0, st>>>(a);
    if (tiles_k > 0) attn_dkv_kernel<T, D><<<dim3((unsigned)(tiles_k * a.parts)), dim3(256), 0, st>>>(a);
    if (tiles_k > 0 && a.parts > 1)
        attn_dkv_join_kernel<T><<<dim3((unsigned)(most_tiles(a.tokens_k, a.sequences, kJoinRows) * (a.hq / a.group))), dim3(256), 0, st>>>(a);
    return s24_launch_status();
}
}  // namespace s24_attn

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
    const int64_t tiles_q = most_tiles(shape->tokens_q, shape->sequences, 128) * shape->hq;
    const int64_t tiles_k = most_tiles(shape->tokens_k, shape->sequences, Backward<128>::BK) * shape->hkv;
    S24_REQUIRE(tiles_q <= kMostGroups && tiles_k <= kMostGroups / 8, S24_ERR_SHAPE);
    Problem a = problem_of(shape);
    a.q = rows_of(Q), a.k = rows_of(K), a.v = rows_of(V), a.o = rows_of(O), a.dO = rows_of(dO);
    a.dq = out_of(dQ), a.dk = out_of(dK), a.dv = out_of(dV);
    a.lse = const_cast<float *>(lse), a.stats = static_cast<float2 *>(workspace), a.parts = (int)parts_of(shape);
    a.sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + stats_bytes(shape));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == S24_BF16) return a.d <= 64 ? backward<uint16_t, 64>(a, tiles_k, tiles_q, st) : backward<uint16_t, 128>(a, tiles_k, tiles_q, st);
    return a.d <= 64 ? backward<s24_half, 64>(a, tiles_k, tiles_q, st) : backward<s24_half, 128>(a, tiles_k, tiles_q, st);
}
