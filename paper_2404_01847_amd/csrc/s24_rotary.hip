// Norms of queries and keys for each head, and the rotation of their positions, in one pass; and the gradients of both.
//
// Forward: s24_rotary.h.  Backward, with g = dz turned back and y = x r:  dw_i = sum of g_i y_i over tokens and heads,  dx_i = r (g_i w_i - y_i mean_j(g_j w_j y_j)).
// Bound by memory: each value is read and written once (of a norm's backward pass x is read as well).
#include "s24_rotary.h"

namespace s24_rotary_rows {
struct Strided { uint16_t *p; int64_t token, head; };

struct ForwardArgs {
    Turn t;
    Strided q, k, qo, ko;
    int shares;
    bool back;
};
// Bound by memory: 8192 tokens of 64 + 8 heads of 128 with norms take 48 us, 6.3 TB/s of what they read and write (a plain copy reaches 6.5), with vector instructions issued in 51 % of the
// cycles; 8 x 1024 tokens of 12 + 12 heads of 64 without 13 (4.0, two calls on the same tensors).  729 tokens take 4, which is the launch.  Rows that the attention reads next are
// stored plainly: past the caches the kernel alone gains, but this and the attention of 8192 tokens of 64 heads on 8 together take 1134 us and not 1088.  Gradients, which a large
// product reads much later, go past them.
template <typename T, int LANES, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary_kernel(const ForwardArgs a)
{
    __shared__ __align__(16) Angles angles[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    const int token = (int)(item / a.shares), share = (int)(item - (int64_t)token * a.shares);
    if (token >= a.t.tokens) return;
    Part<T, LANES, NEIGHBOURS> part(a.t, lane, (lds_angles *)&angles[wave]);
    uint16_t *const qo = a.qo.p + token * a.qo.token, *const ko = a.ko.p + token * a.ko.token;
    turned_rows(a.t, part, a.q.p + token * a.q.token, a.q.head, a.k.p + token * a.k.token, a.k.head, token, share, a.shares, a.back, lane, [&](bool keys, int head, const float (&x)[16]) {
        if (!part.in || head >= (keys ? a.t.hkv : a.t.hq)) return;
        uint16_t *const to = keys ? ko + head * a.ko.head : qo + head * a.qo.head;
        if (a.back) part.template store<true>(to, x);
        else part.store(to, x);
    });
}

// Backward where something is normalised.  A wave has the queries or the keys alone: a stretch of their groups of rows, token by token, over which it sums dw in registers; a
// workgroup's sums go to memory, for another launch to add in order.
// Bound by memory: 8192 tokens of 64 + 8 heads of 128 take 91 us, 5.0 TB/s (adding two tensors of that size to a third, by an elementwise kernel that does nothing else, 5.8), with vector
// instructions issued in 50 % of the cycles at three waves a SIMD: dw keeps 16 sums in each lane, so there are registers for four.  A second group of rows ahead of the arithmetic, two
// groups at once, and seven or eight waves with what they spill, were slower.
struct BackwardArgs {
    Turn t;
    Strided dzq, dzk, xq, xk, dxq, dxk;
    float *sums;           // [q_blocks + k_blocks][d]
    float *dwq, *dwk;
    float beta;
    int q_blocks, k_blocks;
};
template <typename T, int LANES, bool NEIGHBOURS>
__global__ __launch_bounds__(256, 4) void rotary_bwd_kernel(const BackwardArgs a)
{
    using P = Part<T, LANES, NEIGHBOURS>;
    __shared__ float sums[4][16 * LANES];
    __shared__ __align__(16) Angles angles[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool keys = (int)blockIdx.x >= a.q_blocks;
    const int heads = keys ? a.t.hkv : a.t.hq, groups = (heads + P::ROWS - 1) / P::ROWS;
    const Strided &dz = keys ? a.dzk : a.dzq, &x = keys ? a.xk : a.xq, &dx = keys ? a.dxk : a.dxq;
    const uint16_t *const w = keys ? a.t.wk : a.t.wq;
    // Groups of rows are dealt to the waves one by one.  (A stretch of its own for each wave reads from as many places at once as there are waves: 8192 tokens of 64 + 8 heads of 128, both
    // passes, 169 us with whole tokens to a wave, 164 so.)
    const int waves = 4 * (keys ? a.k_blocks : a.q_blocks), mine = 4 * ((int)blockIdx.x - (keys ? a.q_blocks : 0)) + wave, tokens_on = waves / groups, groups_on = waves - tokens_on * groups;
    int token = mine / groups, group = mine - token * groups, of = -1;
    P part(a.t, lane, (lds_angles *)&angles[wave]);
    float by[16], dw[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) by[i] = dw[i] = 0.0f;
    if (w != nullptr && part.in) P::widen(part.load(w), by);
    auto loads = [&](Pieces &p, Pieces &q) {
        const int head = group * P::ROWS + part.r;
        const bool live = part.in && head < heads;
        p = live ? part.load(dz.p + token * dz.token + head * dz.head) : Pieces{};
        q = live && w != nullptr ? part.load(x.p + token * x.token + head * x.head) : Pieces{};
    };
    Pieces next_g{}, next_x{};
    int32_t next_position = 0;
    if (token < a.t.tokens) loads(next_g, next_x), next_position = part.position(a.t, token);
    while (token < a.t.tokens) {
        const Pieces now_g = next_g, now_x = next_x;
        const int32_t position = next_position;
        const int this_token = token, head = group * P::ROWS + part.r;
        group += groups_on, token += tokens_on;
        if (group >= groups) group -= groups, ++token;
        if (token < a.t.tokens) loads(next_g, next_x), next_position = part.position(a.t, token);
        if (of != this_token) part.angles(a.t, position, true, lane), of = this_token;
        float g[16];
        P::widen(now_g, g);
        part.turn(g);
        if (w != nullptr) {
            float y[16];
            P::widen(now_x, y);
            const float r = head < heads ? part.factor(a.t, y) : 0.0f;   // (lanes without a row have zeros, of which the root has no value where eps is 0)
            float mean = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                y[i] *= r;
                dw[i] = fmaf(g[i], y[i], dw[i]);
                g[i] *= by[i];
                mean = fmaf(g[i], y[i], mean);
            }
            mean = row_sum<LANES>(mean) * a.t.share;
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = r * fmaf(-y[i], mean, g[i]);
        }
        if (part.in && head < heads) part.template store<true>(dx.p + this_token * dx.token + head * dx.head, g);
    }
    if (w == nullptr) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int s = LANES; s < 64; s <<= 1) dw[i] += __shfl_xor(dw[i], s);
        if (lane < LANES) sums[wave][16 * lane + i] = dw[i];
    }
    __syncthreads();
    // in the order of the head's values
    for (int v = threadIdx.x; v < 16 * LANES; v += 256) {
        const int i = v & 15;
        const int j = v >> 4;
        const bool apart = 16 * j < a.t.rotated && !NEIGHBOURS;
        const int at = apart ? 8 * j + (i & 7) + (i < 8 ? 0 : a.t.rotated >> 1) : v;
        if (16 * j < a.t.d) a.sums[(int64_t)blockIdx.x * a.t.d + at] = (sums[0][v] + sums[1][v]) + (sums[2][v] + sums[3][v]);
    }
}
// dw = beta dw + the workgroups' sums: a workgroup has sixteen values of the queries' weights or of the keys', and 256 lanes for each four, so that what they wait for is
// few trips to memory.  (Of 519 workgroups 2.4 us, with 64 lanes and one value at a time 3.1; of 4097 7.3 and 7.6.)
__global__ __launch_bounds__(1024) void rotary_dw_kernel(const BackwardArgs a)
{
    __shared__ f32x4 sums[256][4];
    const int sixteens = a.t.d >> 4, keys = (int)blockIdx.x >= sixteens, first = 16 * ((int)blockIdx.x - (keys ? sixteens : 0)), quad = threadIdx.x & 3, row = threadIdx.x >> 2;
    float *const dw = keys ? a.dwk : a.dwq;
    if (dw == nullptr) return;
    const int count = keys ? a.k_blocks : a.q_blocks;
    const float *const from = a.sums + (int64_t)(keys ? a.q_blocks : 0) * a.t.d + first + 4 * quad;
    f32x4 sum = {};
#pragma unroll 8
    for (int i = row; i < count; i += 256) sum += *reinterpret_cast<const f32x4 *>(from + (int64_t)i * a.t.d);
    sums[row][quad] = sum;
    __syncthreads();
    if (threadIdx.x >= 256) return;
    const int v = threadIdx.x >> 4, part = threadIdx.x & 15;   // sixteen lanes to a value
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < 256; i += 16) all += sums[i + part][v >> 2][v & 3];
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) all += __shfl_xor(all, s);
    if (part != 0) return;
    float *const to = dw + first + v;
    *to = a.beta == 0.0f ? all : fmaf(a.beta, *to, all);
}

// ------------------------------------------------------------------ host
static Strided strided(const s24_heads *v) { return v == nullptr ? Strided{} : Strided{static_cast<uint16_t *>(v->data), v->token, v->head}; }

template <typename T> static void rotate(const ForwardArgs &a, bool neighbours, dim3 grid, hipStream_t st)
{
    const dim3 block(256);
    if (a.t.d <= 64) {
        if (neighbours) rotary_kernel<T, 4, true><<<grid, block, 0, st>>>(a);
        else rotary_kernel<T, 4, false><<<grid, block, 0, st>>>(a);
    } else {
        if (neighbours) rotary_kernel<T, 8, true><<<grid, block, 0, st>>>(a);
        else rotary_kernel<T, 8, false><<<grid, block, 0, st>>>(a);
    }
}
template <typename T> static void gradients(const BackwardArgs &a, bool neighbours, dim3 grid, hipStream_t st)
{
    const dim3 block(256);
    if (a.t.d <= 64) {
        if (neighbours) rotary_bwd_kernel<T, 4, true><<<grid, block, 0, st>>>(a);
        else rotary_bwd_kernel<T, 4, false><<<grid, block, 0, st>>>(a);
    } else {
        if (neighbours) rotary_bwd_kernel<T, 8, true><<<grid, block, 0, st>>>(a);
        else rotary_bwd_kernel<T, 8, false><<<grid, block, 0, st>>>(a);
    }
}
static int launch_forward(const Turn &t, const Strided (&x)[4], bool neighbours, bool back, s24_dtype dt, void *stream)
{
    ForwardArgs a{t, x[0], x[1], x[2], x[3], shares_of_token(t.tokens, t.hq, t.hkv, t.d), back};
    const int64_t groups = ((int64_t)t.tokens * a.shares + 3) / 4;
    S24_REQUIRE(groups <= kMostGroups, S24_ERR_SHAPE);
    const dim3 grid((unsigned)groups);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == S24_BF16) rotate<uint16_t>(a, neighbours, grid, st);
    else rotate<s24_half>(a, neighbours, grid, st);
    return s24_launch_status();
}
// Workgroups that share the rows of the queries (the keys): up to sixteen a compute unit for both, with four groups of rows to a wave at least.  (No more than fit a compute unit
// at once leave the last ones to end alone: 8192 tokens of 64 + 8 heads of 128, both passes, with four a compute unit 162 us, with eight 151, sixteen 150, 32 151.)
struct Blocks { int q, k; };
static Blocks blocks_of(int64_t tokens, int64_t hq, int64_t hkv, int64_t d)
{
    const int rows = d <= 64 ? 16 : 8;
    const int64_t q = tokens * ((hq + rows - 1) / rows), k = tokens * ((hkv + rows - 1) / rows), most = 16 * (int64_t)s24_cu_count();
    auto blocks = [&](int64_t items) {
        const int64_t fit = (items + 15) / 16, share = q + k > 0 ? (most * items + q + k - 1) / (q + k) : 0;
        return (int)(fit < share ? fit : share);
    };
    return {blocks(q), blocks(k)};
}
}  // namespace s24_rotary_rows

using namespace s24_rotary_rows;

extern "C" int s24_rotary_fwd(const s24_rotary *rotary, const int32_t *positions, const s24_heads *Q, const s24_heads *K, const s24_heads *Qo, const s24_heads *Ko, int64_t tokens,
                              int64_t hq, int64_t hkv, int64_t d, s24_dtype dt, void *stream)
{
    S24_TRY(check_rotary(rotary, positions, tokens, hq, hkv, d, dt));
    if (hq > 0) S24_TRY(check_rows(Q, tokens, hq, d, false));
    if (hq > 0) S24_TRY(check_rows(Qo, tokens, hq, d, true));
    if (hkv > 0) S24_TRY(check_rows(K, tokens, hkv, d, false));
    if (hkv > 0) S24_TRY(check_rows(Ko, tokens, hkv, d, true));
    if (tokens == 0 || hq + hkv == 0) return S24_OK;
    return launch_forward(turn_args(rotary, positions, tokens, hq, hkv, d), {strided(Q), strided(K), strided(Qo), strided(Ko)}, rotary->interleaved != 0, false, dt, stream);
}

extern "C" int64_t s24_rotary_bwd_workspace(const s24_rotary *rotary, int64_t tokens, int64_t hq, int64_t hkv, int64_t d)
{
    if (rotary == nullptr || (rotary->wq == nullptr && rotary->wk == nullptr) || tokens <= 0 || hq < 0 || hkv < 0 || d <= 0) return 0;
    const Blocks n = blocks_of(tokens, hq, hkv, d);
    return ((int64_t)n.q + n.k) * d * 4;
}

extern "C" int s24_rotary_bwd(const s24_rotary *rotary, const int32_t *positions, const s24_heads *dQo, const s24_heads *dKo, const s24_heads *Q, const s24_heads *K,
                              const s24_heads *dQ, const s24_heads *dK, float *dwq, float *dwk, float beta, int64_t tokens, int64_t hq, int64_t hkv, int64_t d, void *workspace,
                              int64_t workspace_bytes, s24_dtype dt, void *stream)
{
    S24_TRY(check_rotary(rotary, positions, tokens, hq, hkv, d, dt));
    S24_REQUIRE(beta == 0.0f || beta == 1.0f, S24_ERR_SHAPE);
    const bool norm_q = rotary->wq != nullptr && hq > 0, norm_k = rotary->wk != nullptr && hkv > 0;
    for (const bool keys : {false, true}) {
        const int64_t heads = keys ? hkv : hq;
        if (heads == 0) continue;
        S24_TRY(check_rows(keys ? dKo : dQo, tokens, heads, d, false));
        S24_TRY(check_rows(keys ? dK : dQ, tokens, heads, d, true));
        if (keys ? norm_k : norm_q) S24_TRY(check_rows(keys ? K : Q, tokens, heads, d, false));
    }
    S24_REQUIRE((!norm_q || dwq != nullptr) && (!norm_k || dwk != nullptr), S24_ERR_NULL);
    S24_REQUIRE(s24_aligned(dwq, 4) && s24_aligned(dwk, 4) && s24_aligned(workspace, 16), S24_ERR_ALIGN);
    const int64_t need = s24_rotary_bwd_workspace(rotary, tokens, hq, hkv, d);
    S24_REQUIRE(workspace != nullptr || need == 0, S24_ERR_NULL);
    S24_REQUIRE(workspace_bytes >= need, S24_ERR_SHAPE);
    const Turn t = turn_args(rotary, positions, tokens, hq, hkv, d);
    const bool neighbours = rotary->interleaved != 0;
    if (rotary->wq == nullptr && rotary->wk == nullptr) {
        if (tokens == 0 || hq + hkv == 0) return S24_OK;
        return launch_forward(t, {strided(dQo), strided(dKo), strided(dQ), strided(dK)}, neighbours, true, dt, stream);
    }
    const Blocks n = blocks_of(tokens, hq, hkv, d);
    const BackwardArgs a{t, strided(dQo), strided(dKo), strided(Q), strided(K), strided(dQ), strided(dK), static_cast<float *>(workspace), t.wq != nullptr ? dwq : nullptr,
                         t.wk != nullptr ? dwk : nullptr, beta, n.q, n.k};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (n.q + n.k > 0) {
        const dim3 grid((unsigned)(n.q + n.k));
        if (dt == S24_BF16) gradients<uint16_t>(a, neighbours, grid, st);
        else gradients<s24_half>(a, neighbours, grid, st);
    }
    rotary_dw_kernel<<<dim3((unsigned)(d / 8)), dim3(1024), 0, st>>>(a);
    return s24_launch_status();
}
