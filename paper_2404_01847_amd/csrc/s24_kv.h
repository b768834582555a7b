// The paged key-value cache as the kernels see it.
//
// Layout of a page, for one of its key-value heads:  K [page][d], a token's key in one piece;  V [page / E][d][E] with E = 8 tokens for 16-bit
// values and 16 for 8-bit ones: 16 bytes are E consecutive tokens of one channel.  Both products of the attention of a token are matrix
// instructions whose contracted axis lies along a lane's 16 bytes: the channels of K, the tokens of V.  So both go from memory to registers in
// 16-byte loads with nothing in between.
// 8 bits: x ~ s n with n = -127 .. 127 held as n + 128, s = max(max|x| / 127, 2^-126) in fp32 for each token and head.
#pragma once
#include "s24_attn.h"

namespace s24_kv {
using namespace s24_attn;

struct Cache {
    unsigned char *k, *v;
    float *ks, *vs;   // [pages][hkv][page]
    int64_t pages;
    int page, shift, hkv, d;   // page = 1 << shift
};
struct Strided { uint16_t *p; int64_t token, head; };

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

// ---- host
inline int check_cache(const s24_kv_cache *c, s24_dtype dt)
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
inline Cache cache_of(const s24_kv_cache *c)
{
    return {static_cast<unsigned char *>(c->K), static_cast<unsigned char *>(c->V), c->k_step, c->v_step, c->pages, (int)c->page,
            __builtin_ctzll((unsigned long long)c->page), (int)c->hkv, (int)c->d};
}
}  // namespace s24_kv
