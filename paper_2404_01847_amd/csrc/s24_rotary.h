// Heads as rows that are normalised and turned by their token's position, for the kernels that do so on the way (training, the cache).
//
// y_i = x_i w_i r with r = (mean x^2 + eps)^-1/2, or y = x;  a pair (a, b) of y turned by its angle: (a cos - b sin, b cos + a sin).
// A lane has eight pairs of a row: 16 bytes of their first values and 16 of their second (or both in one piece of 32, where neighbours are pairs), so that a row of d
// values is d / 16 lanes, each pair lies within a lane, and all is moved in pieces of 16 bytes.
#pragma once
#include "s24_attn.h"

namespace s24_rotary_rows {
using namespace s24_attn;

struct Turn {
    const int32_t *positions;    // [axes][tokens]
    const double *frequencies;   // [rotated / 2]: radians for each step of the position
    const int32_t *axis;         // [rotated / 2], or NULL: all pairs turn by the first
    const uint16_t *wq, *wk;     // [d], or NULL: not normalised
    float eps, share;            // 1 / d
    int axes, rotated, d, tokens, hq, hkv;
};

// Cosine and sine of a fraction of a turn in 32 bits.  An eighth of a turn to either side of a multiple of a quarter: there the Taylor series to the 9th and 8th power are
// within 2e-9 and 3e-8.
__device__ __forceinline__ void turn_of(uint32_t phase, float &cosine, float &sine)
{
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(phase - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
    const float u = x * x;
    const float s = fmaf(x * u, fmaf(u, fmaf(u, fmaf(u, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -0.166666667f), x);
    const float c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, 2.48015873e-5f, -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.0f);
    const float p = quarter & 1 ? s : c, q = quarter & 1 ? c : s;
    cosine = __uint_as_float(__float_as_uint(p) ^ ((quarter + 1) & 2) << 30);
    sine = __uint_as_float(__float_as_uint(q) ^ (quarter & 2) << 30);
}

// Of x what is left of whole turns, as a word of 64 bits
__device__ __forceinline__ uint64_t turn_word(double x)
{
    const double steps = (x - rint(x)) * 0x1p32, whole = fmin(floor(steps), 2147483647.0);
    return ((uint64_t)(uint32_t)(int32_t)whole << 32) + (uint32_t)fmin((steps - whole) * 0x1p32, 4294967295.0);
}
// A frequency's fraction of a turn in 64 bits, for frequencies up to 2^40 within 3 of its last places: 1 / (2 pi) in two doubles, and what the product with the first
// leaves.  (The product rounded to one double would be off by 2^-53 of the frequency, which the position multiplies: 100 radians a step are off by 2e-5 radians at position 2^31 so.)
__device__ __forceinline__ uint64_t turn_fraction(double frequency)
{
#pragma clang fp contract(off)
    const double turns = frequency * 0x1.45f306dc9c883p-3, left = fma(frequency, 0x1.45f306dc9c883p-3, -turns);
    return turn_word(turns) + turn_word(fma(frequency, -9.839338337591243e-18, left));
}

// Sum over the lanes of a row
template <int LANES> __device__ __forceinline__ float row_sum(float x)
{
    static_assert(LANES == 4 || LANES == 8, "a row's lanes");
#if defined(__HIP_DEVICE_COMPILE__)
    auto moved = [](float v, auto control) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(control)::value, 0xf, 0xf, true)); };
    x += moved(x, std::integral_constant<int, 0xB1>());                     // lanes 1 0 3 2 of four
    x += moved(x, std::integral_constant<int, 0x4E>());                     // 2 3 0 1
    if (LANES == 8) x += moved(x, std::integral_constant<int, 0x141>());    // eight, the other way round
#endif
    return x;
}
// Largest of their magnitudes, compared as bits: what is no number is the largest of all
template <int LANES> __device__ __forceinline__ uint32_t row_max(uint32_t x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));
    if (LANES == 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));
#endif
    return x;
}

struct Pieces { uint4 a, b; };
// Cosines and sines of a token's pairs, of a wave
struct Angles { float cosine[64], sine[64]; };
typedef __attribute__((address_space(3))) Angles lds_angles;
// The 16 values of a lane, and how they are paired
template <typename T, int LANES, bool NEIGHBOURS> struct Part {
    static constexpr int ROWS = 64 / LANES;   // that a wave has at a time
    int j, r, a, b;    // lane of a row, row; where its two pieces start
    bool in, turned;   // whether it has values, and whether they are turned
    float cosine[8], sine[8];
    // The pair that the lane finds the angle of: its frequency as a fraction of a turn, high + low / 2^32 in 2^-32, and where its axis has the positions
    uint32_t high, low;
    bool none;         // it has no value: neither has the pair
    const int32_t *at;
    lds_angles *shared;
    __device__ __forceinline__ Part(const Turn &t, int lane, lds_angles *angles)
    {
        j = lane & (LANES - 1), r = lane / LANES, shared = angles;
        in = 16 * j < t.d, turned = 16 * j < t.rotated;
        const bool apart = turned && !NEIGHBOURS;
        a = apart ? 8 * j : 16 * j, b = apart ? (t.rotated >> 1) + 8 * j : 16 * j + 8;
        high = low = 0, none = false, at = t.positions;
        if (2 * lane >= t.rotated) return;
        if (t.axis != nullptr) at += (int64_t)min((uint32_t)t.axis[lane], (uint32_t)t.axes - 1) * t.tokens;
        const double frequency = t.frequencies[lane];
        const uint64_t word = turn_fraction(frequency);
        high = (uint32_t)(word >> 32), low = (uint32_t)word;
        none = !(fabs(frequency) < (double)INFINITY);
    }
    // The angles of a token: each lane has one, and its row's eight come from the others'.  Of the frequency's fraction of a turn in 64
    // bits times the position whole turns fall out of the word, and what the fraction is off by becomes 2^-31 of a turn at most.
    __device__ __forceinline__ void angles(const Turn &t, int32_t position, bool back, int lane)
    {
        if (t.rotated == 0) return;
        const uint32_t n = (uint32_t)position;
        float c, s;
        turn_of(n * high + __umulhi(n, low) - (position < 0 ? low : 0), c, s);
        if (none) c = s = NAN;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        shared->cosine[lane] = c, shared->sine[lane] = back ? -s : s;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const lds_byte *from = (const lds_byte *)shared + 32 * j;
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            const f32x4 x = __builtin_bit_cast(f32x4, lds_load(from + 4 * e)), y = __builtin_bit_cast(f32x4, lds_load(from + 256 + 4 * e));
#pragma unroll
            for (int i = 0; i < 4; ++i) cosine[e + i] = x[i], sine[e + i] = y[i];
        }
    }
    // Position of a token on the lane's axis
    __device__ __forceinline__ int32_t position(const Turn &t, int token) const { return t.rotated > 0 ? at[token] : 0; }
    __device__ __forceinline__ Pieces load(const uint16_t *row) const
    {
        return {*reinterpret_cast<const uint4 *>(row + a), *reinterpret_cast<const uint4 *>(row + b)};
    }
    static __device__ __forceinline__ void widen(const Pieces &p, float (&x)[16])
    {
        using Num = s24_num<T>;
        const uint32_t w[8] = {p.a.x, p.a.y, p.a.z, p.a.w, p.b.x, p.b.y, p.b.z, p.b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[2 * i] = Num::lo(w[i]), x[2 * i + 1] = Num::hi(w[i]);
    }
    template <bool PAST = false> __device__ __forceinline__ void store(uint16_t *row, const float (&x)[16]) const
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
        const uint4 first = make_uint4(w[0], w[1], w[2], w[3]), second = make_uint4(w[4], w[5], w[6], w[7]);
        if (PAST) {
            s24_store_stream(row + a, first), s24_store_stream(row + b, second);
        } else {
            *reinterpret_cast<uint4 *>(row + a) = first;
            *reinterpret_cast<uint4 *>(row + b) = second;
        }
    }
    // 1 / sqrt(mean x^2 + eps) of the row
    __device__ __forceinline__ float factor(const Turn &t, const float (&x)[16]) const
    {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
        sum = row_sum<LANES>(in ? sum : 0.0f);
        const float mean = fmaf(sum, t.share, t.eps), y = __builtin_amdgcn_rsqf(mean);
        return y * fmaf(-0.5f * mean * y, y, 1.5f);   // (the estimate and a Newton step: a few tenths of a step more exact)
    }
    __device__ __forceinline__ void turn(float (&x)[16]) const
    {
        if (!turned) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = NEIGHBOURS ? 2 * e : e, q = NEIGHBOURS ? 2 * e + 1 : 8 + e;
            const float u = x[p], v = x[q];
            x[p] = fmaf(u, cosine[e], -v * sine[e]), x[q] = fmaf(v, cosine[e], u * sine[e]);
        }
    }
};

// Rows of a token's heads, ROWS at a time, queries before keys: a wave takes every `shares`-th such group from `share` on, the next one's loads ahead of this one's
// arithmetic.  use(keys, head, x): the row of a lane, turned; `head` is past the last one for lanes that have none.
template <typename P, typename Use>
__device__ __forceinline__ void turned_rows(const Turn &t, P &part, const uint16_t *q, int64_t q_head, const uint16_t *k, int64_t k_head, int token, int share, int shares, bool back, int lane, Use use)
{
    const int of_q = (t.hq + P::ROWS - 1) / P::ROWS, all = of_q + (t.hkv + P::ROWS - 1) / P::ROWS;
    if (share >= all) return;
    auto load = [&](int group) {
        const bool keys = group >= of_q;
        const int head = (keys ? group - of_q : group) * P::ROWS + part.r;
        return part.in && head < (keys ? t.hkv : t.hq) ? part.load(keys ? k + head * k_head : q + head * q_head) : Pieces{};
    };
    auto weights = [&](bool keys) {
        const uint16_t *w = keys ? t.wk : t.wq;
        return w != nullptr && part.in ? part.load(w) : Pieces{};
    };
    Pieces next = load(share), w = weights(share >= of_q);
    part.angles(t, part.position(t, token), back, lane);
    for (int group = share; group < all; group += shares) {
        const Pieces now = next;
        const bool keys = group >= of_q;
        if (keys && group - shares < of_q && group != share) w = weights(true);
        if (group + shares < all) next = load(group + shares);
        float x[16];
        P::widen(now, x);
        if ((keys ? t.wk : t.wq) != nullptr) {
            float by[16];
            P::widen(w, by);
            const float f = part.factor(t, x);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= f * by[i];
        }
        part.turn(x);
        use(keys, (keys ? group - of_q : group) * P::ROWS + part.r, x);
    }
}

// ---- host
inline int check_rotary(const s24_rotary *r, const int32_t *positions, int64_t tokens, int64_t hq, int64_t hkv, int64_t d, s24_dtype dt)
{
    S24_REQUIRE(r != nullptr, S24_ERR_NULL);
    S24_REQUIRE(s24_valid_dtype(dt), S24_ERR_DTYPE);
    S24_REQUIRE(tokens >= 0 && tokens < INT32_MAX / 2 && hq >= 0 && hkv >= 0 && hq < 65536 && hkv < 65536, S24_ERR_SHAPE);
    S24_REQUIRE(d >= 16 && d % 16 == 0 && r->rotated >= 0 && r->rotated % 16 == 0 && r->rotated <= d, S24_ERR_SHAPE);
    S24_REQUIRE(r->axes >= 1 && r->axes <= 65535 && r->eps >= 0.0f && r->eps <= 3.0e38f, S24_ERR_SHAPE);
    S24_REQUIRE(dt != S24_F32 && d <= 128, S24_ERR_UNSUPPORTED);
    if (r->rotated > 0) S24_REQUIRE(r->frequencies != nullptr && (positions != nullptr || tokens == 0), S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(r->frequencies, 8) && s24_aligned(r->axis, 4) && s24_aligned(positions, 4) && s24_aligned(r->wq, 16) && s24_aligned(r->wk, 16), S24_ERR_ALIGN);
    return S24_OK;
}
inline Turn turn_args(const s24_rotary *r, const int32_t *positions, int64_t tokens, int64_t hq, int64_t hkv, int64_t d)
{
    return {positions, r->frequencies, r->axis, static_cast<const uint16_t *>(r->wq), static_cast<const uint16_t *>(r->wk), r->eps, 1.0f / (float)d,
            (int)r->axes, (int)r->rotated, (int)d, (int)tokens, (int)hq, (int)hkv};
}
// Waves that share a token's groups of rows: three groups to a wave at most, fewer where there are too few tokens for sixteen waves a compute unit.  (All of a token's in one
// wave leave the last waves of a launch long ones: 13868 tokens of 64 + 8 heads of 128 appended in 8 bits 114 us so, 106 with four to a wave, 106 with three, 105 with two, 119 with one;
// 8192 tokens of them normalised and turned 51, 49, 49, 50 and 59; 5338 tokens of 20 + 20 heads of 64 appended 27, 27, 24, 24 and 26.)
inline int shares_of_token(int64_t tokens, int64_t hq, int64_t hkv, int64_t d)
{
    const int rows = d <= 64 ? 16 : 8;
    const int64_t groups = (hq + rows - 1) / rows + (hkv + rows - 1) / rows, fill = tokens > 0 ? 16 * (int64_t)s24_cu_count() / tokens : 1, third = (groups + 2) / 3;
    const int64_t most = fill > third ? fill : third;
    return (int)(most < 1 ? 1 : most > groups ? groups : most);
}
}  // namespace s24_rotary_rows
