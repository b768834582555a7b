// The paged key-value cache: tokens written to it (in 8 bits: quantised), sequences read back, and attention of one new token over it.
//
// Layout of a page, for one of its key-value heads:  K [page][d], a token's key in one piece;  V [page / E][d][E] with E = 8 tokens for 16-bit
// values and 16 for 8-bit ones: 16 bytes are E consecutive tokens of one channel.  Both products of the attention of a token are matrix
// instructions whose contracted axis lies along a lane's 16 bytes: the channels of K, the tokens of V.  So both go from memory to registers in
// 16-byte loads with nothing in between.
// 8 bits: x ~ s n with n = -127 .. 127 held as n + 128, s = max(max|x| / 127, 2^-126) in fp32 for each token and head.
#include "s24_attn.h"

#include <math.h>

namespace s24_kv {
using namespace s24_attn;

struct Cache {
    unsigned char *k, *v;
    float *ks, *vs;   // [pages][hkv][page]
    int64_t pages;
    int page, shift, hkv, d;   // page = 1 << shift
};
struct Strided { uint16_t *p; int64_t token, head; };

// n nearest to x / s, ties to even, exactly: the estimate is at most one off, and x - n s is exact in fp32 for 16-bit x (a multiple of the last
// place of s, and no larger than s).
__device__ __forceinline__ int nearest(float x, float s, float inverse)
{
    const float n = rintf(x * inverse), twice = 2.0f * fmaf(-n, s, x);
    const int i = (int)n, odd = i & 1;
    return i + (twice > s || (twice == s && odd)) - (twice < -s || (twice == -s && odd));
}

// ------------------------------------------------------------------ writing
struct WriteArgs {
    Cache c;
    Strided k, v;
    const int64_t *places;
    int tokens;
};
// Sixteen tokens of a page that follow each other, of one head (PAIR: of two, d <= 64): row r of 16 lanes has the tokens 4r .. 4r + 3, a lane eight channels of
// them from `c` on.
template <bool PAIR> struct Lane {
    int r, c, h;
    bool live;
    __device__ __forceinline__ Lane(const Cache &cache, int unit, int lane)
    {
        r = lane >> 4, c = 8 * (PAIR ? lane & 7 : lane & 15), h = PAIR ? 2 * unit + (lane >> 3 & 1) : unit;
        live = c < cache.d && h < cache.hkv;
    }
};
// Magnitudes are compared as the bits that they are, two at a time: what is no number is the largest of all, and stays.
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Largest of the lanes that hold a token of a head
template <bool PAIR> __device__ __forceinline__ uint32_t token_max(uint32_t x)
{
#if defined(__HIP_DEVICE_COMPILE__)
    x = larger(x, __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true));    // lanes 1 0 3 2 of four
    x = larger(x, __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true));    // 2 3 0 1
    x = larger(x, __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));   // eight, the other way round
    if (!PAIR) x = larger(x, __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));   // sixteen
#endif
    return x;
}
// The step of a token whose magnitudes have these two as their largest: NaN if one of them is none or is infinite, so that nothing finite comes of it
template <typename T> __device__ __forceinline__ float step_for(uint32_t two)
{
    const float most = s24_num<T>::lo(max(two & 0xFFFFu, two >> 16));
    return most < INFINITY ? fmaxf(__fdiv_rn(most, 127.0f), 0x1p-126f) : NAN;
}
// The whole numbers + 128 of eight values, each in the low byte: rounded by adding what pushes the fraction out, and where one lies so close to
// the middle of two that the product's own rounding could decide, taken again exactly.
template <typename T> __device__ __forceinline__ void eight_numbers(uint4 packed, float step, float inverse, uint32_t (&n)[8])
{
    using Num = s24_num<T>;
    constexpr float kPush = 12582912.0f + 128.0f;
    const uint32_t w[4] = {packed.x, packed.y, packed.z, packed.w};
    float x[8], off = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = i & 1 ? Num::hi(w[i >> 1]) : Num::lo(w[i >> 1]);
        const float pushed = fmaf(x[i], inverse, kPush);
        n[i] = __float_as_uint(pushed);
        off = fmaxf(off, fabsf(fmaf(x[i], inverse, kPush - pushed)));
    }
    if (__any(off > 0.49997f)) {   // 127 times the error of the inverse is below 2.2e-5
#pragma unroll
        for (int i = 0; i < 8; ++i) n[i] = (uint32_t)(nearest(x[i], step, inverse) + 128);
    }
}
template <typename T, bool PAIR> __device__ __forceinline__ float step_of(uint4 x)
{
    const uint32_t sign = 0x7FFF7FFFu;
    return step_for<T>(token_max<PAIR>(larger(larger(x.x & sign, x.y & sign), larger(x.z & sign, x.w & sign))));
}

// Many tokens: a wave looks at sixteen of them and takes, of K or of V, those runs that begin there and lie within sixteen aligned places of a page, one after
// the other.  Of a prompt, whatever place it starts at, that is sixteen tokens to a wave: V then leaves in pieces of 16 bytes.  Where more than two runs begin in
// the sixteen tokens (new tokens of many sequences) all of them are taken at once, and V leaves value by value: 1280 tokens of 8 heads of 128 that do not follow each other take
// 14 us in 8 bits so, 33 run by run (16 bits: 13 and 16), 16384 of them 160 and 180.  (At once from two runs on, runs of 8 tokens gain another 5 % and prompts in 16 bits lose as much.)
// Bound by memory: 17408 tokens of 8 heads of 128 take 27 us in 8 bits and 33 in 16 (4.0 and 4.3 TB/s; a plain copy of as many bytes reaches 5.7).  Stores past
// the caches, in whole lines, take 25 and 31; but the reading back that follows then takes longer by more: both together 44 us with these, 50 with those.
template <typename T, int BITS, bool PAIR>
__global__ __launch_bounds__(256) void kv_write_runs_kernel(const WriteArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int units = PAIR ? (a.c.hkv + 1) / 2 : a.c.hkv, item = 4 * blockIdx.x + wave, window = (item >> 1) / units;
    const bool values = item & 1;
    const Lane<PAIR> at(a.c, (item >> 1) - window * units, lane);
    const int first_token = 16 * window;
    if (first_token >= a.tokens) return;
    const Strided from = values ? a.v : a.k;
    const int mine = first_token - 1 + lane;   // lanes 0 .. 33: the token before, the window, and as many as a run that begins in it may reach
    const int64_t place = mine >= 0 && mine < a.tokens && lane < 34 ? a.places[mine] : -1;
    const int64_t before = __shfl_up(place, 1);
    const uint64_t starts = __ballot(mine >= a.tokens || mine <= 0 || (place & 15) == 0 || place != before + 1) >> 1;
    const uint32_t runs = (uint32_t)starts & (0xFFFFu >> max(16 - (a.tokens - first_token), 0));
    if (__popc(runs) > 2) {   // their tokens at once, each to its own place
        const int first_run = __builtin_ctz(runs), last_run = 31 - __builtin_clz(runs), end = last_run + __builtin_ctzll(starts >> (last_run + 1)) + 1;
        for (int base = 0; base < end; base += 16) {
            uint4 x[4];
            int64_t to[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = base + 4 * at.r + i;
                to[i] = __shfl(place, k + 1);
                if (!at.live || k < first_run || k >= end || to[i] >= a.c.pages << a.c.shift) to[i] = -1;
                x[i] = to[i] >= 0 ? *reinterpret_cast<const uint4 *>(from.p + (int64_t)(first_token + k) * from.token + at.h * from.head + at.c) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t first = ((to[i] >> a.c.shift) * a.c.hkv + at.h) << a.c.shift;   // of the page, in tokens of one head
                const int in = (int)(to[i] & (a.c.page - 1));
                if constexpr (BITS == 16) {
                    if (to[i] < 0) continue;
                    if (!values) {
                        *reinterpret_cast<uint4 *>(a.c.k + ((first + in) * a.c.d + at.c) * 2) = x[i];
                        continue;
                    }
                    uint16_t *v = reinterpret_cast<uint16_t *>(a.c.v) + first * a.c.d + ((int64_t)(in >> 3) * a.c.d + at.c) * 8 + (in & 7);
                    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                } else {
                    uint32_t bytes[8];
                    const float step = step_of<T, PAIR>(x[i]);
                    eight_numbers<T>(x[i], step, __builtin_amdgcn_rcpf(step), bytes);
                    if (to[i] < 0) continue;
                    if (at.c == 0) (values ? a.c.vs : a.c.ks)[first + in] = step;
                    if (!values) {
                        *reinterpret_cast<uint2 *>(a.c.k + (first + in) * a.c.d + at.c) =
                            make_uint2(four_bytes(bytes[0], bytes[1], bytes[2], bytes[3]), four_bytes(bytes[4], bytes[5], bytes[6], bytes[7]));
                        continue;
                    }
                    unsigned char *v = a.c.v + first * a.c.d + ((int64_t)(in >> 4) * a.c.d + at.c) * 16 + (in & 15);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[16 * e] = (unsigned char)bytes[e];
                }
            }
        }
        return;
    }
    for (uint32_t left = runs; left != 0; left &= left - 1) {
        const int j = __builtin_ctz(left), token = first_token + j;
        if (token >= a.tokens) break;
        const int n = __builtin_ctzll(starts >> (j + 1)) + 1;
        const int64_t to = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(place >> 32), j + 1) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)place, j + 1));
        if (to < 0 || to >= a.c.pages << a.c.shift) continue;
        const int skip = (int)(to & 15);
        const int64_t base = ((((to >> a.c.shift) * a.c.hkv + at.h) << a.c.shift) + (to & (a.c.page - 1) & ~15));   // of the sixteen, in tokens of one head
        uint4 x[4];
        bool live[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = 4 * at.r + i - skip;
            live[i] = at.live && k >= 0 && k < n;
            x[i] = live[i] ? *reinterpret_cast<const uint4 *>(from.p + (int64_t)(token + k) * from.token + at.h * from.head + at.c) : make_uint4(0, 0, 0, 0);
        }
        if constexpr (BITS == 16) {
            if (!values) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (live[i]) *reinterpret_cast<uint4 *>(a.c.k + ((base + 4 * at.r + i) * a.c.d + at.c) * 2) = x[i];
                continue;
            }
            uint32_t lo[8], hi[8];   // of a channel: tokens 4r, 4r + 1 and 4r + 2, 4r + 3
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[4];   // channels 2i and 2i + 1 of the four tokens
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = i == 0 ? x[k].x : i == 1 ? x[k].y : i == 2 ? x[k].z : x[k].w;
                lo[2 * i] = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u), lo[2 * i + 1] = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
                hi[2 * i] = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u), hi[2 * i + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
            }
            uint16_t *v = reinterpret_cast<uint16_t *>(a.c.v) + base * a.c.d + ((int64_t)(at.r >> 1) * a.c.d + at.c) * 8;
            if (n == 16) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {   // even rows get channel e of both, odd rows channel e + 4
                    swap_rows(lo[e], lo[e + 4]), swap_rows(hi[e], hi[e + 4]);
                    if (at.live) *reinterpret_cast<uint4 *>(v + 8 * (e + 4 * (at.r & 1))) = make_uint4(lo[e], hi[e], lo[e + 4], hi[e + 4]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (live[i]) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[8 * e + 4 * (at.r & 1) + i] = (uint16_t)((i < 2 ? lo[e] : hi[e]) >> (16 * (i & 1)));
                    }
            }
        } else {
            uint32_t bytes[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float step = step_of<T, PAIR>(x[i]);
                eight_numbers<T>(x[i], step, __builtin_amdgcn_rcpf(step), bytes[i]);
                if (live[i] && at.c == 0) (values ? a.c.vs : a.c.ks)[base + 4 * at.r + i] = step;
            }
            if (!values) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (live[i])
                        *reinterpret_cast<uint2 *>(a.c.k + (base + 4 * at.r + i) * a.c.d + at.c) =
                            make_uint2(four_bytes(bytes[i][0], bytes[i][1], bytes[i][2], bytes[i][3]), four_bytes(bytes[i][4], bytes[i][5], bytes[i][6], bytes[i][7]));
                continue;
            }
            unsigned char *v = a.c.v + base * a.c.d + at.c * 16;
            if (n == 16) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {   // row r gets all sixteen tokens of channel 4*half + r
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = four_bytes(bytes[0][4 * half + e], bytes[1][4 * half + e], bytes[2][4 * half + e], bytes[3][4 * half + e]);
                    transpose_rows(w);
                    if (at.live) *reinterpret_cast<uint4 *>(v + 16 * (4 * half + at.r)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (live[i]) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[16 * e + 4 * at.r + i] = (unsigned char)bytes[i][e];
                    }
            }
        }
    }
}

// Few tokens, in any order: a wave takes one token of one head, a lane two channels.  V is written value by value.  Bound by the launch.
template <typename T, int BITS>
__global__ __launch_bounds__(256) void kv_write_kernel(const WriteArgs a)
{
    using Num = s24_num<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    if (item >= (int64_t)a.tokens * a.c.hkv) return;
    const int token = (int)(item / a.c.hkv), h = (int)(item - (int64_t)token * a.c.hkv);
    const int64_t place = a.places[token];
    if (place < 0 || place >= a.c.pages << a.c.shift) return;
    const int64_t first = ((place >> a.c.shift) * a.c.hkv + h) << a.c.shift;   // of the page, in tokens of one head
    const int at = (int)(place & (a.c.page - 1)), i = 2 * lane;
    const bool live = i < a.c.d;
    uint32_t xk = 0, xv = 0;
    if (live) {
        xk = *reinterpret_cast<const uint32_t *>(a.k.p + token * a.k.token + h * a.k.head + i);
        xv = *reinterpret_cast<const uint32_t *>(a.v.p + token * a.v.token + h * a.v.head + i);
    }
    if (BITS == 16) {
        if (!live) return;
        *reinterpret_cast<uint32_t *>(a.c.k + ((first + at) * a.c.d + i) * 2) = xk;
        uint16_t *v = reinterpret_cast<uint16_t *>(a.c.v) + first * a.c.d + ((int64_t)(at >> 3) * a.c.d + i) * 8 + (at & 7);
        v[0] = (uint16_t)xv, v[8] = (uint16_t)(xv >> 16);
    } else {
        uint32_t mk = xk & 0x7FFF7FFFu, mv = xv & 0x7FFF7FFFu;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) mk = larger(mk, __shfl_xor(mk, s)), mv = larger(mv, __shfl_xor(mv, s));
        const float sk = step_for<T>(mk), sv = step_for<T>(mv);
        const float ik = __builtin_amdgcn_rcpf(sk), iv = __builtin_amdgcn_rcpf(sv);
        if (lane == 0) a.c.ks[first + at] = sk, a.c.vs[first + at] = sv;
        if (!live) return;
        *reinterpret_cast<uint16_t *>(a.c.k + (first + at) * a.c.d + i) =
            (uint16_t)((nearest(Num::lo(xk), sk, ik) + 128) | (nearest(Num::hi(xk), sk, ik) + 128) << 8);
        unsigned char *v = a.c.v + first * a.c.d + ((int64_t)(at >> 4) * a.c.d + i) * 16 + (at & 15);
        v[0] = (unsigned char)(nearest(Num::lo(xv), sv, iv) + 128), v[16] = (unsigned char)(nearest(Num::hi(xv), sv, iv) + 128);
    }
}

// ------------------------------------------------------------------ reading back
struct ReadArgs {
    Cache c;
    Strided k, v;
    const int *table, *cu;
    int64_t width;
    int sequences, tokens;
};
// Sixteen tokens of a sequence by a wave, four waves a workgroup, arranged in its lanes as in the writing of runs.
// Bound by memory: 17408 tokens of 8 heads of 128 take 27 us in 8 bits and 32 in 16 (4.0 and 4.4 TB/s).  Stores past the caches take 24 and 30, but then the
// attention that reads the rows next takes longer by more: read and 512 queries of each of 4 sequences 148 us with these, 163 with those.
template <typename T, int BITS, bool PAIR>
__global__ __launch_bounds__(256) void kv_read_kernel(const ReadArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int units = PAIR ? (a.c.hkv + 1) / 2 : a.c.hkv, tile = blockIdx.x / units;
    const Lane<PAIR> at(a.c, blockIdx.x - tile * units, lane);
    int sequence, index, count;
    if (!find_tile(a.cu, a.sequences, a.tokens, 64, tile, lane, sequence, index, count)) return;
    const Span s = span(a.cu, sequence, a.tokens);
    const int pos = index * 64 + 16 * wave, n = min(s.count - pos, 16);
    if (n <= 0 || pos >> a.c.shift >= a.width) return;
    const uint32_t id = min((uint32_t)a.table[sequence * a.width + (pos >> a.c.shift)], (uint32_t)a.c.pages - 1);
    const int64_t base = (((int64_t)id * a.c.hkv + at.h) << a.c.shift) + (pos & (a.c.page - 1));
    if (!at.live) return;   // (the lanes that exchange parts below are live together)
    struct Four { uint32_t w[4]; };   // eight values
    Four xk[4], xv[4];
    if constexpr (BITS == 16) {
        const uint16_t *v = reinterpret_cast<const uint16_t *>(a.c.v) + base * a.c.d + ((int64_t)(at.r >> 1) * a.c.d + at.c) * 8;
        uint32_t lo[8], hi[8];   // of a channel: tokens 4r, 4r + 1 and 4r + 2, 4r + 3
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            xk[e] = __builtin_bit_cast(Four, *reinterpret_cast<const uint4 *>(a.c.k + ((base + 4 * at.r + e) * a.c.d + at.c) * 2));
            const uint4 x = *reinterpret_cast<const uint4 *>(v + 8 * (e + 4 * (at.r & 1)));
            lo[e] = x.x, hi[e] = x.y, lo[e + 4] = x.z, hi[e + 4] = x.w;
            swap_rows(lo[e], lo[e + 4]), swap_rows(hi[e], hi[e + 4]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                xv[i].w[e] = __builtin_amdgcn_perm(i < 2 ? lo[2 * e + 1] : hi[2 * e + 1], i < 2 ? lo[2 * e] : hi[2 * e], i & 1 ? 0x07060302u : 0x05040100u);
    } else {
        const f32x4 sk = *reinterpret_cast<const f32x4 *>(a.c.ks + base + 4 * at.r), sv = *reinterpret_cast<const f32x4 *>(a.c.vs + base + 4 * at.r);
        uint2 nk[4];
        uint32_t x[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) nk[i] = *reinterpret_cast<const uint2 *>(a.c.k + (base + 4 * at.r + i) * a.c.d + at.c);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint4 v = *reinterpret_cast<const uint4 *>(a.c.v + base * a.c.d + (at.c + 4 * half + at.r) * 16);
            x[half][0] = v.x, x[half][1] = v.y, x[half][2] = v.z, x[half][3] = v.w;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) transpose_rows(x[half]);   // now of channel 4*half + e the tokens 4r .. 4r + 3
        auto value = [](uint32_t w, int byte) { return (float)(w >> (8 * byte) & 255u) - 128.0f; };
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = e < 2 ? nk[i].x : nk[i].y;
                xk[i].w[e] = pack2<T>(value(w, 2 * (e & 1)) * sk[i], value(w, 2 * (e & 1) + 1) * sk[i]);
                xv[i].w[e] = pack2<T>(value(x[e >> 1][2 * (e & 1)], i) * sv[i], value(x[e >> 1][2 * (e & 1) + 1], i) * sv[i]);
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (4 * at.r + i >= n) continue;
        const int64_t t = s.first + pos + 4 * at.r + i;
        *reinterpret_cast<uint4 *>(a.k.p + t * a.k.token + at.h * a.k.head + at.c) = __builtin_bit_cast(uint4, xk[i]);
        *reinterpret_cast<uint4 *>(a.v.p + t * a.v.token + at.h * a.v.head + at.c) = __builtin_bit_cast(uint4, xv[i]);
    }
}

// ------------------------------------------------------------------ attention of one new token
struct DecodeArgs {
    Cache c;
    Strided q, o;
    const int *table, *lengths;
    int64_t width;
    int sequences, hq, group, sixteens, shares;   // sixteens: of query heads in a group; shares: of the positions of all sequences, for each of the heads
    float scale;
    bool whole;    // a share is a sequence
    float *part;   // [2 shares][hq][d + 4]: sums, reference, weight, and two unused
};
__device__ __forceinline__ int length_of(const DecodeArgs &a, int b) { return min(max(a.lengths[b], 0), (int)(a.width << a.c.shift)); }
// The sequences' blocks of 64 positions lie one after the other and are shared out evenly, whatever sequences they belong to: share p has blocks p*each ..
// (p + 1)*each - 1 of them.  A sequence that lies within one share is finished there.  Of others each share leaves the sums of its part: at 2p if the sequence
// starts no later than the share, at 2p + 1 otherwise (a share has one such part at either end, at most).
__device__ __forceinline__ int blocks_of(int length) { return (length + 63) >> 6; }
// The blocks of 256 sequences, four to a lane: for more than 64, whose lengths else lie one to a lane.  (Looked through 64 at a time instead, 600 sequences cost
// a launch 10 us.)
struct Lists {
    int n[4], sum;
    __device__ __forceinline__ Lists(const DecodeArgs &a, int base, int lane)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = base + 4 * lane + i < a.sequences ? blocks_of(length_of(a, base + 4 * lane + i)) : 0;
        sum = n[0] + n[1] + n[2] + n[3];
    }
};

// Sixteen bytes of the cache as operands of 8 channels (tokens) each
__device__ __forceinline__ uint4 halves(uint32_t a, uint32_t b)
{
    // a byte under the exponent of 1024 is 1024 + byte
    auto two = [](uint32_t x, uint32_t select) {
        const f16x2 v = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(x, 0x64646464u, select));
        return __builtin_bit_cast(uint32_t, v - (f16x2){(_Float16)1152.0f, (_Float16)1152.0f});
    };
    return make_uint4(two(a, 0x00050004u), two(a, 0x00070006u), two(b, 0x00050004u), two(b, 0x00070006u));
}

// A wave takes a share of the positions for one key-value head and 16 of its query heads, in blocks of 64; the four of a workgroup know nothing of each other.
// Bound by memory where the cache is large: 8 sequences of 60000 to 65536 positions, 64 heads on 8 of 128 in 8 bits, take 177 us (5.9 TB/s of 6.6 that a large copy
// reaches); 128 ragged sequences, 20 heads of 64 in 8 bits, 75 us (5.7); 16 ragged ones, 32 heads of 128 in 16 bits, 37 us (4.7), of which 5 add the parts.
// One of 1000 positions is bound by two launches and the way from a length to a page number to the page: 10.5 us.  As many waves as the device holds have one share
// each, so that none waits for another and few parts are left.  (In the launch itself, by the wave that comes last, the parts are added in 13.0 us where it was 11.4
// for the one sequence, and in 38.1 where it was 37.5 for the 16: what a wave of another XCD wrote has to be waited for either way.)
// Of a block, S^T = K Q^T has positions as rows: row 4g + r of tile t is position 16g + 4t + r, so that a lane's
// weights are those of 16 consecutive positions, which is what it holds of V.
// Softmax in 8 bits: the weights go to the product as exp(s - ref) * (step of V) in binary16, where ref has the largest step so far as a factor too, so that
// they stay at 2^9 or less; the factor is in the sum of the weights as well and cancels.  (A step below 2^-100 counts as that, for ref to stay in range.)
// Heads of every size have a kernel of their own, in which the addresses within a page are constants.  (With those of 64 and 128 for all, 32 sequences of 4096 positions,
// 32 heads on 8 in 16 bits, take 98 us for heads of 96 and 92 for 80; so 74 and 72.)
constexpr float kRise = 8.0f;   // as in the forward pass over packed sequences: how far a score may exceed the reference before it moves
template <typename T, int D, int BITS>
__global__ __launch_bounds__(256, 2) void attn_decode_kernel(const DecodeArgs a)
{
    using M = typename std::conditional<BITS == 8, s24_half, T>::type;   // the products of an 8-bit cache are binary16: it holds -127 .. 127
    using Num = s24_num<T>;
    constexpr int KL = BITS == 8 ? (D + 63) / 64 : (D + 31) / 32, VL = BITS == 8 ? 1 : 2;   // 16-byte loads of a key; of a channel's positions
    constexpr int QL = BITS == 8 ? 2 * KL : KL;   // operands of a query
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    constexpr int d = D;
    const int heads = a.c.hkv * a.sixteens, item = 4 * blockIdx.x + wave, share = item / heads, which = item - share * heads;
    const int h = which / a.sixteens, q0 = 16 * (which - h * a.sixteens), mine = min(16, a.group - q0);   // of the group's query heads
    if (share >= a.shares) return;
    struct Cursor { int b, first, pos, length; };   // a block: its sequence, which has `first` as its first block; the position at which it starts
    auto advance = [&](Cursor c) {
        c.pos += 64;
        if (c.pos < c.length) return c;
        c.first += blocks_of(c.length), c.pos = 0;
        do {   // there is one more: only blocks of the share are asked for
            c.length = __builtin_amdgcn_readfirstlane(length_of(a, ++c.b));
        } while (c.length == 0);
        return c;
    };
    int each, begin, steps;
    Cursor now{share, 0, 0, 0};
    if (a.whole) {
        now.length = __builtin_amdgcn_readfirstlane(length_of(a, share));
        each = steps = blocks_of(now.length), begin = 0;
        if (steps == 0)
            for (int i = lane; i < mine * (d >> 3); i += 64) {
                const int n = i / (d >> 3);
                *reinterpret_cast<uint4 *>(a.o.p + share * a.o.token + (h * a.group + q0 + n) * a.o.head + 8 * (i - n * (d >> 3))) = make_uint4(0, 0, 0, 0);
            }
    } else if (a.sequences <= 64) {
        const int length = lane < a.sequences ? length_of(a, lane) : 0, n = blocks_of(length), sum = running_sum(n), total = __builtin_amdgcn_readlane(sum, 63);
        each = (total + a.shares - 1) / a.shares, begin = share * each, steps = min(total - begin, each);
        now.b = steps > 0 ? __ffsll((unsigned long long)__ballot(begin < sum)) - 1 : 0;
        now.first = __builtin_amdgcn_readlane(sum - n, now.b), now.length = __builtin_amdgcn_readlane(length, now.b);
    } else {
        Lists lists(a, 0, lane);
        int total = lists.sum;
        for (int base = 256; base < a.sequences; base += 256) total += Lists(a, base, lane).sum;
        total = __builtin_amdgcn_readlane(running_sum(total), 63);   // below 2^31, as the host has seen to
        each = (total + a.shares - 1) / a.shares, begin = share * each, steps = min(total - begin, each);
        for (int base = 0, before = 0; base < a.sequences && steps > 0; base += 256) {
            if (base > 0) lists = Lists(a, base, lane);
            const int sum = running_sum(lists.sum);
            const unsigned long long past = __ballot(begin < before + sum);
            if (past == 0) {
                before += __builtin_amdgcn_readlane(sum, 63);
                continue;
            }
            const int owner = __ffsll(past) - 1, b = base + 4 * owner;
            now.first = before + __builtin_amdgcn_readlane(sum - lists.sum, owner), now.b = b;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const int n = __builtin_amdgcn_readlane(lists.n[i], owner);
                if (now.b == b + i && begin >= now.first + n) now.first += n, ++now.b;
            }
            now.length = __builtin_amdgcn_readfirstlane(length_of(a, now.b));
            break;
        }
    }
    if (steps <= 0) return;
    now.pos = 64 * (begin - now.first);

    // Positions 16*(col/4) .. of a block for K, 16*g .. for V: each sixteen lie in one page.
    constexpr int token = d * (BITS / 8);   // bytes of a token of one head
    const uint32_t page_tokens = (uint32_t)a.c.hkv << a.c.shift;
    const unsigned char *const lane_k = a.c.k + ((int64_t)h << a.c.shift) * token + (col & 3) * token, *const lane_v = a.c.v + ((int64_t)h << a.c.shift) * token;
    struct Place { int64_t k, v; };   // in tokens of one head
    auto place = [&](const Cursor &at) {
        const int *table = a.table + at.b * a.width;
        auto of = [&](int group) {
            const int pos = min(at.pos + 16 * group, (at.length - 1) & ~15);
            const uint32_t id = min((uint32_t)table[pos >> a.c.shift], (uint32_t)a.c.pages - 1);
            return (int64_t)((uint64_t)id * page_tokens) + (pos & (a.c.page - 1));
        };
        return Place{of(col >> 2), of(g)};
    };
    uint4 fk[4][KL], fv[D / 16][VL];
    f32x4 sk[4], sv[4];
    auto load_k = [&](Place p) {
        const unsigned char *row = lane_k + p.k * token;
        const float *step = a.c.ks + ((int64_t)h << a.c.shift) + p.v;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int k = 0; k < KL; ++k)
                fk[t][k] = s24_load_stream(row + 4 * t * token + 16 * (64 * k + 64 <= token ? 4 * k + g : min(4 * k + g, (token >> 4) - 1)));   // (past it the query has zeros)
            if (BITS == 8) sk[t] = *reinterpret_cast<const f32x4 *>(step + 4 * t);
        }
    };
    auto load_v = [&](Place p) {
        const unsigned char *page = lane_v + p.v * token;
        const float *step = a.c.vs + ((int64_t)h << a.c.shift) + p.v;
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (BITS == 8) sv[t] = *reinterpret_cast<const f32x4 *>(step + 4 * t);
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
#pragma unroll
            for (int u = 0; u < VL; ++u)
                fv[n][u] = s24_load_stream(page + (u * d + 16 * n + col) * 16);
    };
    // the queries, an operand of 16 columns
    uint4 q[QL];
    float c = 0.0f;
    auto load_q = [&](int b) {
        const uint16_t *row = a.q.p + b * a.q.token + (h * a.group + q0 + min(col, mine - 1)) * a.q.head;
        float most = 0.0f;
        c = a.scale * kLog2e;
#pragma unroll
        for (int k = 0; k < QL; ++k) {
            const int i = BITS == 8 ? 64 * (k >> 1) + 16 * g + 8 * (k & 1) : 32 * k + 8 * g;
            q[k] = i < d && col < mine ? *reinterpret_cast<const uint4 *>(row + i) : make_uint4(0, 0, 0, 0);
        }
        if (BITS == 8) {   // scaled by a power of two into what binary16 holds
            const uint32_t *x = reinterpret_cast<const uint32_t *>(q);
#pragma unroll
            for (int i = 0; i < 4 * QL; ++i) most = fmaxf(most, fmaxf(fabsf(Num::lo(x[i])), fabsf(Num::hi(x[i]))));
            most = column_max(most);
            const int e = most > 0.0f ? ilogbf(most) : 0;
            uint32_t y[4 * QL];
#pragma unroll
            for (int i = 0; i < 4 * QL; ++i) y[i] = pack2<s24_half>(ldexpf(Num::lo(x[i]), -e), ldexpf(Num::hi(x[i]), -e));
#pragma unroll
            for (int k = 0; k < QL; ++k) q[k] = make_uint4(y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]);
            c = ldexpf(c, e);
        }
    };
    // (Past the caches: a step reads its cache once, and other layers' caches before it comes back.  On caches that are not there anyway 8 x 60000 positions
    // in 8 bits take 178 us instead of 197, 16 ragged sequences of 32 heads 37 instead of 40; a single one of 1000 positions 11.2 instead of 10.5.)
    // The loads run ahead: the keys of the next block are requested as soon as this one's scores are formed, its values as soon as they are summed, and the
    // page numbers a block before that.
    Cursor ahead = now;
    Place next{};
    {
        const Place first = place(now);
        if (steps > 1) ahead = advance(now), next = place(ahead);
        load_k(first), load_v(first);
        load_q(now.b);
    }
    float m, rise, wide, l;   // reference; its part from the steps of V, which are at most `wide`; sum of the weights
    f32x4 o[D / 16];
    auto clear = [&] {
        m = -1e30f, rise = BITS == 8 ? -100.0f : 0.0f, wide = 0x1p-100f, l = 0.0f;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) o[n] = f32x4{};
    };
    clear();
    for (int i = 0; i < steps; ++i) {
        const Place coming = next;
        const Cursor after = ahead;
        if (i + 2 < steps) ahead = advance(ahead), next = place(ahead);
        const int k0 = now.pos, end = now.length;
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4{};
#pragma unroll
            for (int k = 0; k < KL; ++k) {
                if constexpr (BITS == 8) {
                    s[t] = mma<M>(halves(fk[t][k].x, fk[t][k].y), q[2 * k], s[t]);
                    s[t] = mma<M>(halves(fk[t][k].z, fk[t][k].w), q[2 * k + 1], s[t]);
                } else
                    s[t] = mma<M>(fk[t][k], q[k], s[t]);
            }
            if (BITS == 8) s[t] *= sk[t];
        }
        if (i + 1 < steps) load_k(coming);
        if (k0 + 64 > end) {   // what lies past the sequence's end may hold anything
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool in = k0 + 16 * g + 4 * t + r < end;
                    s[t][r] = in ? s[t][r] : -INFINITY;
                    if (BITS == 8) sv[t][r] = in ? sv[t][r] : 0.0f;
                }
            if (BITS == 16) {
#pragma unroll
                for (int n = 0; n < D / 16; ++n)
#pragma unroll
                    for (int u = 0; u < VL; ++u) {
                        uint32_t *x = reinterpret_cast<uint32_t *>(&fv[n][u]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int left = end - (k0 + 16 * g + 8 * u + 2 * j);
                            x[j] = left >= 2 ? x[j] : left == 1 ? x[j] & 0xFFFFu : 0u;
                        }
                    }
            }
        }
        float top = s[0][0], step = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, s[t][r]);
            if (BITS == 8) step = fmaxf(step, fmaxf(fmaxf(sv[t][0], sv[t][1]), fmaxf(sv[t][2], sv[t][3])));
        }
        top *= c;
        if (__any(top > m - rise + kRise || (BITS == 8 && step > wide))) {   // m - rise: the reference of the scores alone
            if (BITS == 8) {
                step = column_max(step);
                if (step > wide) wide = 2.0f * step;
            }
            const float lift = BITS == 8 ? __builtin_amdgcn_logf(wide) : 0.0f, now_m = fmaxf(m - rise, column_max(top)) + lift;
            const float shrink = __builtin_amdgcn_exp2f(m - now_m);
            m = now_m, rise = lift, l *= shrink;
#pragma unroll
            for (int n = 0; n < D / 16; ++n) o[n] *= shrink;
        }
        uint4 p[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], c, -m));
                l += s[t][r];
                if (BITS == 8) s[t][r] *= sv[t][r];
            }
#pragma unroll
        for (int u = 0; u < 2; ++u) p[u] = operand<M>(s[2 * u], s[2 * u + 1]);
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            if constexpr (BITS == 8) {
                o[n] = mma<M>(halves(fv[n][0].x, fv[n][0].y), p[0], o[n]);
                o[n] = mma<M>(halves(fv[n][0].z, fv[n][0].w), p[1], o[n]);
            } else {
                o[n] = mma<M>(fv[n][0], p[0], o[n]);
                o[n] = mma<M>(fv[n][1], p[1], o[n]);
            }
        }
        if (i + 1 < steps) load_v(coming);

        if (k0 + 64 < end && i + 1 < steps) {   // more of this sequence
            now = after;
            continue;
        }
        l = column_sum(l);
        const int head = h * a.group + q0 + col;
        if (now.first >= begin && now.first + blocks_of(end) <= begin + each) {
            const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
            uint16_t *out = a.o.p + now.b * a.o.token + head * a.o.head;
            if (col < mine) {
#pragma unroll
                for (int n = 0; n < D / 16; ++n)
                    *reinterpret_cast<uint2 *>(out + 16 * n + 4 * g) =
                        make_uint2(pack2<T>(o[n][0] * inverse, o[n][1] * inverse), pack2<T>(o[n][2] * inverse, o[n][3] * inverse));
            }
        } else {
            float *to = a.part + ((int64_t)(2 * share + (now.first > begin)) * a.hq + head) * (d + 4);
            if (col < mine) {
#pragma unroll
                for (int n = 0; n < D / 16; ++n)
                    *reinterpret_cast<f32x4 *>(to + 16 * n + 4 * g) = o[n];
                if (g == 0) *reinterpret_cast<float2 *>(to + d) = make_float2(m, l);
            }
        }
        if (i + 1 < steps) {
            now = after;
            clear();
            load_q(now.b);
        }
    }
}

// The parts of a sequence that lies in more than one share, added: WAVES waves a query head, a lane two channels, a wave every WAVES-th part.
// A sequence of no positions, which no share has, gets its zeros.
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void attn_join_kernel(const DecodeArgs a)
{
    __shared__ float4 waves[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = a.c.d;
    const int item = WAVES == 4 ? blockIdx.x : 4 * blockIdx.x + wave, b = item / a.hq, head = item - b * a.hq;
    if (b >= a.sequences) return;
    const int e = min(2 * lane, d - 2);
    int total = 0, first = 0, blocks;   // of all sequences, of those before this one, of this one
    if (a.sequences <= 64) {
        const int n = lane < a.sequences ? blocks_of(length_of(a, lane)) : 0, sum = running_sum(n);
        total = __builtin_amdgcn_readlane(sum, 63), blocks = __builtin_amdgcn_readlane(n, b), first = __builtin_amdgcn_readlane(sum, b) - blocks;
    } else {
        for (int base = 0; base < a.sequences; base += 256) {
            const Lists lists(a, base, lane);
            total += lists.sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) first += base + 4 * lane + i < b ? lists.n[i] : 0;
        }
        total = __builtin_amdgcn_readlane(running_sum(total), 63), first = __builtin_amdgcn_readlane(running_sum(first), 63);
        blocks = blocks_of(length_of(a, b));
    }
    const int last = first + blocks - 1;
    uint32_t *out = reinterpret_cast<uint32_t *>(a.o.p + b * a.o.token + head * a.o.head + e);
    if (last < first) {
        if ((WAVES == 1 || wave == 0) && 2 * lane < d) *out = 0;
        return;
    }
    const int each = (total + a.shares - 1) / a.shares, p0 = first / each, count = last / each - p0 + 1;
    if (count == 1) return;
    const int64_t step = 2 * (int64_t)a.hq * (d + 4);
    const float *part = a.part + p0 * step + (int64_t)head * (d + 4);
    const float *part0 = first > p0 * each ? part + (step >> 1) : part;   // of the first share, where the sequence may start late
    // References and sums in one trip to memory: what the sums are taken to moves with the largest reference so far.  (With a trip for the references before it, one
    // sequence of 1000 positions of 32 heads of 128 takes 11.1 us instead of 10.5.)
    constexpr int AT_ONCE = 4;
    float ref = -INFINITY, x = 0.0f, y = 0.0f, w = 0.0f;
    for (int i = WAVES == 4 ? wave : 0; i < count; i += WAVES * AT_ONCE) {
        float2 of[AT_ONCE], v[AT_ONCE];
        float top = ref;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int at = min(i + u * WAVES, count - 1);
            const float *from = at == 0 ? part0 : part + at * step;
            of[u] = *reinterpret_cast<const float2 *>(from + d), v[u] = *reinterpret_cast<const float2 *>(from + e);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            of[u].x = i + u * WAVES < count ? of[u].x : -INFINITY;
            top = fmaxf(top, of[u].x);
        }
        const float shrink = __builtin_amdgcn_exp2f(ref - top);
        ref = top, x *= shrink, y *= shrink, w *= shrink;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const float f = __builtin_amdgcn_exp2f(of[u].x - ref);
            const bool in = i + u * WAVES < count;
            x = fmaf(f, in ? v[u].x : 0.0f, x), y = fmaf(f, in ? v[u].y : 0.0f, y), w = fmaf(f, in ? of[u].y : 0.0f, w);
        }
    }
    if constexpr (WAVES == 4) {
        waves[wave][lane] = make_float4(x, y, w, ref);
        __syncthreads();
        if (wave != 0) return;
        float4 of[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) of[i] = waves[i][lane];
        const float top = fmaxf(fmaxf(of[0].w, of[1].w), fmaxf(of[2].w, of[3].w));
        x = y = w = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = __builtin_amdgcn_exp2f(of[i].w - top);
            x = fmaf(f, of[i].x, x), y = fmaf(f, of[i].y, y), w = fmaf(f, of[i].z, w);
        }
    }
    const float inverse = w == 0.0f ? 0.0f : 1.0f / w;
    if (2 * lane < d) *out = pack2<T>(x * inverse, y * inverse);
}

// ------------------------------------------------------------------ host
static int check_cache(const s24_kv_cache *c, s24_dtype dt)
{
    S24_REQUIRE(c != nullptr, S24_ERR_NULL);
    S24_REQUIRE(s24_valid_dtype(dt), S24_ERR_DTYPE);
    S24_REQUIRE(c->bits == 16 || c->bits == 8, S24_ERR_DTYPE);
    S24_REQUIRE(c->pages >= 0 && c->pages < INT32_MAX && c->hkv > 0 && c->hkv < 65536, S24_ERR_SHAPE);
    S24_REQUIRE(c->page >= 16 && c->page <= 1 << 16 && (c->page & (c->page - 1)) == 0, S24_ERR_SHAPE);
    S24_REQUIRE(c->d >= 16 && c->d % 16 == 0, S24_ERR_SHAPE);
    S24_REQUIRE(dt != S24_F32 && c->d <= 128, S24_ERR_UNSUPPORTED);
    if (c->pages > 0) S24_REQUIRE(c->K != nullptr && c->V != nullptr && (c->bits == 16 || (c->k_step != nullptr && c->v_step != nullptr)), S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(c->K, 16) && s24_aligned(c->V, 16) && s24_aligned(c->k_step, 16) && s24_aligned(c->v_step, 16), S24_ERR_ALIGN);
    return S24_OK;
}
static Cache cache_of(const s24_kv_cache *c)
{
    return {static_cast<unsigned char *>(c->K), static_cast<unsigned char *>(c->V), c->k_step, c->v_step, c->pages, (int)c->page,
            __builtin_ctzll((unsigned long long)c->page), (int)c->hkv, (int)c->d};
}
static Strided strided(const s24_heads *v) { return {static_cast<uint16_t *>(v->data), v->token, v->head}; }

template <typename T, int BITS> static void write(const WriteArgs &a, bool runs, dim3 grid, hipStream_t st)
{
    const dim3 block(256);
    if (!runs) kv_write_kernel<T, BITS><<<grid, block, 0, st>>>(a);
    else if (a.c.d <= 64) kv_write_runs_kernel<T, BITS, true><<<grid, block, 0, st>>>(a);
    else kv_write_runs_kernel<T, BITS, false><<<grid, block, 0, st>>>(a);
}
template <typename T, int BITS> static void read(const ReadArgs &a, dim3 grid, hipStream_t st)
{
    const dim3 block(256);
    if (a.c.d <= 64) kv_read_kernel<T, BITS, true><<<grid, block, 0, st>>>(a);
    else kv_read_kernel<T, BITS, false><<<grid, block, 0, st>>>(a);
}

// Shares of the positions for each of `heads` products: as many waves as the device holds at a time.
static int64_t shares_of(int64_t heads, int64_t d)
{
    const int64_t n = (d <= 64 ? 12 : 8) * (int64_t)s24_cu_count() / heads;
    return n < 1 ? 1 : n;
}
}  // namespace s24_kv

using namespace s24_kv;

extern "C" int s24_kv_write(const s24_kv_cache *cache, const s24_heads *K, const s24_heads *V, const int64_t *places, int64_t tokens, s24_dtype dt,
                            void *stream)
{
    S24_TRY(check_cache(cache, dt));
    S24_REQUIRE(tokens >= 0 && tokens < INT32_MAX / 2, S24_ERR_SHAPE);
    S24_TRY(check_rows(K, tokens, cache->hkv, cache->d, false));
    S24_TRY(check_rows(V, tokens, cache->hkv, cache->d, false));
    S24_REQUIRE(places != nullptr || tokens == 0, S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(places, 8), S24_ERR_ALIGN);
    if (tokens == 0 || cache->pages == 0) return S24_OK;
    const WriteArgs a{cache_of(cache), strided(K), strided(V), places, (int)tokens};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // The runs' kernel from 40 tokens of a head for each compute unit on.  (8 bits, 8 heads of 128, both sides: 1024 tokens 7.9 us by runs, 6.1 one by one; 2048
    // tokens 7.6 and 9.5; 16384 tokens 24 and 50.  12 heads of 64, 1024 tokens: 7.3 and 7.2.  16 bits, 8 heads of 128, 1024 tokens: 5.3 and 6.3.  Those are prompts.  Tokens that
    // do not follow each other, which the host does not see, take 14 and 9.5 us at 1280 tokens, 27 and 22 at 4096, 160 and 154 at 16384.)
    const int64_t units = cache->d <= 64 ? (cache->hkv + 1) / 2 : cache->hkv, waves = 2 * ((tokens + 15) / 16) * units;   // of K and of V
    const bool runs = tokens * cache->hkv >= 40 * (int64_t)s24_cu_count();
    const int64_t groups = runs ? (waves + 3) / 4 : (tokens * cache->hkv + 3) / 4;
    S24_REQUIRE((runs ? waves + 3 : groups) <= kMostGroups, S24_ERR_SHAPE);   // (the runs' kernel numbers its waves in an int)
    const dim3 grid((unsigned)groups);
    if (cache->bits == 16) write<uint16_t, 16>(a, runs, grid, st);   // a copy, whatever the type
    else if (dt == S24_BF16) write<uint16_t, 8>(a, runs, grid, st);
    else write<s24_half, 8>(a, runs, grid, st);
    return s24_launch_status();
}

extern "C" int s24_kv_read(const s24_kv_cache *cache, const int32_t *table, int64_t width, const int32_t *cu, int64_t sequences, int64_t tokens,
                           const s24_heads *K, const s24_heads *V, s24_dtype dt, void *stream)
{
    S24_TRY(check_cache(cache, dt));
    S24_REQUIRE(tokens >= 0 && tokens < INT32_MAX / 2 && sequences >= 0 && sequences < INT32_MAX / 2 && width >= 0 && width < INT32_MAX, S24_ERR_SHAPE);
    S24_TRY(check_rows(K, tokens, cache->hkv, cache->d, true));
    S24_TRY(check_rows(V, tokens, cache->hkv, cache->d, true));
    S24_REQUIRE(cu != nullptr && (table != nullptr || width == 0 || sequences == 0), S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(table, 4) && s24_aligned(cu, 4), S24_ERR_ALIGN);
    const int64_t groups = most_tiles(tokens, sequences, 64) * (cache->d <= 64 ? (cache->hkv + 1) / 2 : cache->hkv);
    S24_REQUIRE(groups <= kMostGroups, S24_ERR_SHAPE);
    if (groups == 0 || cache->pages == 0 || width == 0) return S24_OK;
    const ReadArgs a{cache_of(cache), strided(K), strided(V), table, cu, width, (int)sequences, (int)tokens};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups);
    if (cache->bits == 16) read<uint16_t, 16>(a, grid, st);
    else if (dt == S24_BF16) read<uint16_t, 8>(a, grid, st);
    else read<s24_half, 8>(a, grid, st);
    return s24_launch_status();
}

extern "C" int64_t s24_attn_decode_workspace(const s24_kv_cache *cache, int64_t sequences, int64_t hq)
{
    if (cache == nullptr || cache->hkv <= 0 || sequences < 0 || hq <= 0 || hq % cache->hkv != 0) return 0;
    return 2 * shares_of(cache->hkv * ((hq / cache->hkv + 15) / 16), cache->d) * hq * (cache->d + 4) * 4;
}

namespace s24_kv {
template <typename T, int BITS> static void decode(const DecodeArgs &a, dim3 grid, hipStream_t st)
{
    const dim3 block(256);
    switch (a.c.d) {
    case 16: attn_decode_kernel<T, 16, BITS><<<grid, block, 0, st>>>(a); break;
    case 32: attn_decode_kernel<T, 32, BITS><<<grid, block, 0, st>>>(a); break;
    case 48: attn_decode_kernel<T, 48, BITS><<<grid, block, 0, st>>>(a); break;
    case 64: attn_decode_kernel<T, 64, BITS><<<grid, block, 0, st>>>(a); break;
    case 80: attn_decode_kernel<T, 80, BITS><<<grid, block, 0, st>>>(a); break;
    case 96: attn_decode_kernel<T, 96, BITS><<<grid, block, 0, st>>>(a); break;
    case 112: attn_decode_kernel<T, 112, BITS><<<grid, block, 0, st>>>(a); break;
    default: attn_decode_kernel<T, 128, BITS><<<grid, block, 0, st>>>(a); break;
    }
    if (a.whole) return;
    // A wave adds the parts of a row where there are few of them.  (Four and one: 64 sequences of 512 positions, 64 heads on 8 of 128 in 8 bits, 27.6 and 23.9 us;
    // one of 4096 10.6 and 14.7.)
    const int64_t rows = (int64_t)a.sequences * a.hq;
    if (a.shares <= 8 * (int64_t)a.sequences) attn_join_kernel<T, 1><<<dim3((unsigned)((rows + 3) / 4)), block, 0, st>>>(a);
    else attn_join_kernel<T, 4><<<dim3((unsigned)rows), block, 0, st>>>(a);
}
}  // namespace s24_kv

extern "C" int s24_attn_decode(const s24_kv_cache *cache, const s24_heads *Q, int64_t hq, const int32_t *table, int64_t width, const int32_t *lengths,
                               int64_t sequences, float scale, const s24_heads *O, void *workspace, int64_t workspace_bytes, s24_dtype dt, void *stream)
{
    S24_TRY(check_cache(cache, dt));
    S24_REQUIRE(sequences >= 0 && sequences < INT32_MAX / 2 && width >= 0 && width < INT32_MAX && hq > 0 && hq < 65536 && hq % cache->hkv == 0, S24_ERR_SHAPE);
    S24_REQUIRE(width * cache->page <= (int64_t)1 << 30 && sequences * width * cache->page < INT32_MAX, S24_ERR_SHAPE);
    S24_REQUIRE(scale > 0.0f && scale <= 3.0e38f, S24_ERR_SHAPE);
    S24_TRY(check_rows(Q, sequences, hq, cache->d, false));
    S24_TRY(check_rows(O, sequences, hq, cache->d, true));
    if (sequences == 0) return S24_OK;
    S24_REQUIRE(lengths != nullptr && workspace != nullptr && (table != nullptr || width == 0), S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(table, 4) && s24_aligned(lengths, 4) && s24_aligned(workspace, 16), S24_ERR_ALIGN);
    S24_REQUIRE(workspace_bytes >= s24_attn_decode_workspace(cache, sequences, hq), S24_ERR_SHAPE);
    DecodeArgs a{cache_of(cache), strided(Q), strided(O), table, lengths, cache->pages > 0 ? width : 0};
    a.sequences = (int)sequences, a.hq = (int)hq, a.group = (int)(hq / cache->hkv), a.sixteens = (a.group + 15) / 16;
    const int64_t heads = cache->hkv * a.sixteens;
    // (No more than there are blocks: for a few short sequences the host knows of fewer.)
    const int64_t most = sequences * ((a.width * cache->page + 63) / 64), fit = shares_of(heads, cache->d);
    // A wave has whole sequences, and nothing is left to add, where the table holds few positions: up to 128, or 512 if there are as many sequences as shares.
    // (Shared out and whole: one sequence of 128 positions of 12 heads of 64 7.3 and 5.0 us, 8 of 256 8.8 and 10.8; 256 of 64 heads on 8 of 128 in 8 bits, 128
    // positions 39 and 17, 512 positions 71 and 48; 64 of 1024 positions of 32 heads on 8 in 16 bits 55 and 75.)
    a.whole = a.width * cache->page <= (sequences >= fit ? 512 : 128);
    const int64_t shares = a.whole ? sequences : most < fit ? (most > 0 ? most : 1) : fit;
    const int64_t groups = (shares * heads + 3) / 4;
    S24_REQUIRE(sequences * hq <= kMostGroups / 2, S24_ERR_SHAPE);
    a.shares = (int)shares, a.scale = scale, a.part = static_cast<float *>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups);
    if (dt == S24_BF16) cache->bits == 16 ? decode<uint16_t, 16>(a, grid, st) : decode<uint16_t, 8>(a, grid, st);
    else cache->bits == 16 ? decode<s24_half, 16>(a, grid, st) : decode<s24_half, 8>(a, grid, st);
    return s24_launch_status();
}
