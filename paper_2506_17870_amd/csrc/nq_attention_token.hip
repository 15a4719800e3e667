// nq_attention_token: attention of one new token of each sequence over the paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(x_j - m),  x_j = scale log2(e) (q . k_j),  m the largest x so far
//
// Bound by the bytes of the cache's keys and values, each of which is read once, straight into registers in the matrix instructions'
// operand order: S^T = K Q^T of 16 tokens x 32 columns x 16 query heads (those of one key head; a group of fewer leaves columns
// empty, which the matrix core has time for), then O^T = V^T P^T of 32 tokens.  The lane that holds four tokens' scores of a head
// after the first product holds the same tokens' place in the second one's operand, because the order in which a product sums its
// tokens is free: the probabilities never leave their registers, and a lane keeps the maximum and the sum of one head.
#include "nq_attention.h"

namespace nq {

typedef __bf16 at_b8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_h2 __attribute__((ext_vector_type(2)));
typedef float at_f4 __attribute__((ext_vector_type(4)));

constexpr int TK_WAVES = 4, TK_TILE = 32, TK_COLS = 16;   // tokens of a wave's step; query heads of a matrix tile
constexpr float TK_LOG2E = 1.44269504088896340736f;

struct TokenParams {
    const void *q;
    void *o;
    const int32_t *table, *length;
    float *partial;                       // [sequences][q_heads][parts][D + 4]: sums of o, then m and l
    CacheView cache;
    int64_t ldq, ldo, ldtable;
    int32_t sequences, max_length, Hq, Hkv, group, col_tiles, D, parts, target;
    float scale;                          // times log2(e)
};

// How a sequence of `length` tokens is split: into chunks of this many, `parts` at most.  The chunk is the share of a workgroup if
// all tokens of the call were dealt evenly to p.target of them, so that long sequences of a mixed batch go to more workgroups than short ones.
// Every wave that asks makes the same sum.
__device__ __forceinline__ int chunk_of(const TokenParams &p, int length)
{
    if (p.parts == 1) return max(length, 1);
    int64_t total = 0;
    for (int i = threadIdx.x & 63; i < p.sequences; i += 64) total += min(max(p.length[i], 0), p.max_length);
    if (p.sequences > 1) {
#pragma unroll
        for (int k = 1; k < 64; k *= 2) total += __shfl_xor(total, k);
    } else {
        total = __shfl(total, 0);
    }
    const int64_t blocks = (int64_t)p.Hkv * p.col_tiles;
    const int64_t even = (total * blocks + p.target - 1) / p.target;
    const int64_t least = (length + p.parts - 1) / p.parts;
    const int64_t chunk = min(max(max(even, least), (int64_t)(TK_WAVES * TK_TILE)), (int64_t)length + 1);
    return (int)((chunk + TK_TILE - 1) / TK_TILE * TK_TILE);
}

template <typename T>
__device__ __forceinline__ at_f4 mma(uint4 a, uint4 b, at_f4 c)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f8_h8, a), __builtin_bit_cast(f8_h8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(at_b8, a), __builtin_bit_cast(at_b8, b), c, 0, 0, 0);
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_bit_cast(uint32_t, at_h2{(_Float16)a, (_Float16)b});
    else
        return pack_bf16(a, b);
}
template <typename T>
__device__ __forceinline__ float low_of(uint32_t d)
{
    if constexpr (__is_same(T, _Float16))
        return (float)__builtin_bit_cast(at_h2, d)[0];
    else
        return __builtin_bit_cast(float, d << 16);
}
template <typename T>
__device__ __forceinline__ float high_of(uint32_t d)
{
    if constexpr (__is_same(T, _Float16))
        return (float)__builtin_bit_cast(at_h2, d)[1];
    else
        return __builtin_bit_cast(float, d & 0xffff0000u);
}

// Two e4m3 codes (the low or the high half of d) as two values of T; every code is one exactly.
template <typename T, bool HIGH>
__device__ __forceinline__ uint32_t codes2(uint32_t d)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, 1.0f, HIGH));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d, 1.0f, HIGH));
}

// T: queries and outputs; CODES: an e4m3 cache; DP: columns, head_dim rounded up to a form; FAST: head_dim == DP and pages of
// whole 16 tokens, so that a tile of 16 tokens has one page, found by scalar loads.
template <typename T, bool CODES, int DP, bool FAST>
__global__ void __launch_bounds__(TK_WAVES * 64) k_attention_token(const TokenParams p)
{
    constexpr int KJ = DP / 32, VC = DP / 16, ES = CODES ? 1 : 2;      // products to a score; columns of V to a lane
    constexpr int KW = CODES ? 2 : 4;                                   // dwords of eight elements
    using VT = typename std::conditional<CODES, bf16_t, T>::type;       // codes times their scale: bf16's range, in two parts
    __shared__ float joined[2][TK_COLS][DP + 4];
    __shared__ float tops[TK_WAVES][TK_COLS];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int s = blockIdx.z, hk = blockIdx.y / p.col_tiles, col0 = (blockIdx.y - hk * p.col_tiles) * TK_COLS;
    const int cols = min(TK_COLS, p.group - col0), head0 = hk * p.group + col0;
    const int length = min(max(__builtin_amdgcn_readfirstlane(p.length[s]), 0), p.max_length);
    const int chunk = chunk_of(p, length);
    if (blockIdx.x > 0 && (int64_t)blockIdx.x * chunk >= length) return; // (the first part of a sequence without tokens writes its zeros)
    const int begin = blockIdx.x * chunk, end = min(length, begin + chunk);

    uint4 q[KJ];
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
        q[j] = make_uint4(0, 0, 0, 0);
        const int d = 32 * j + 8 * g;
        if (n < cols && d < p.D) __builtin_memcpy(&q[j], static_cast<const T *>(p.q) + s * p.ldq + (int64_t)(head0 + n) * p.D + d, 16);
    }
    const int32_t *table = p.table + s * p.ldtable;
    const int64_t at_head = hk * p.cache.head_step, scale_head = hk * p.cache.scale_head_step;

    at_f4 o[VC];
#pragma unroll
    for (int c = 0; c < VC; ++c) o[c] = at_f4{0, 0, 0, 0};
    float m = -__builtin_inff(), l = 0.0f;
    bool seen = false;

    for (int t0 = begin + wave * TK_TILE; t0 < end; t0 += TK_WAVES * TK_TILE) {
        // ---- keys and values of 32 tokens: token 16 u + n for the first product, 16 u + 4 g + i for the second
        uint32_t k[2][KJ][KW], v[2][4][VC / (4 / ES)];
        float ks[2][4], vs[2][4];
        bool live[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int tu = t0 + 16 * u;
            auto row = [&](int t, bool &ok, int64_t &at, int64_t &scale) {
                ok = t < end;
                const int tc = ok ? t : 0;
                int pg, place;
                if constexpr (FAST) {
                    const int first = tu < end ? tu : 0;
                    pg = (int)divide((uint32_t)first, p.cache.by_page);
                    place = first - pg * (int)p.cache.by_page.d + (ok ? t - tu : 0);
                } else {
                    pg = (int)divide((uint32_t)tc, p.cache.by_page);
                    place = tc - pg * (int)p.cache.by_page.d;
                }
                const int32_t page = table[pg];
                ok = ok && (uint32_t)page < (uint32_t)p.cache.pages;
                at = ok ? (int64_t)page * p.cache.page_step + (int64_t)place * p.cache.token_step + at_head : at_head;
                scale = ok ? (int64_t)page * p.cache.scale_page_step + (int64_t)place * p.cache.scale_token_step + scale_head : scale_head;
            };
            bool ok;
            int64_t at, scale;
            row(tu + n, ok, at, scale);
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                const int d = 32 * j + 8 * g;
                const bool in = FAST || d < p.D;
                uint32_t x[KW];
                __builtin_memcpy(x, p.cache.k + (at + (in ? d : 0)) * ES, sizeof x);
#pragma unroll
                for (int i = 0; i < KW; ++i) k[u][j][i] = in ? x[i] : 0u;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                row(tu + 4 * g + i, ok, at, scale);
                live[u][i] = ok;
                const int d = VC * n;
                const bool in = FAST || d < p.D;
                uint32_t x[VC / (4 / ES)];
                if (FAST || d + VC <= p.D) {
                    __builtin_memcpy(x, p.cache.v + (at + (in ? d : 0)) * ES, sizeof x);
                } else {
#pragma unroll
                    for (int e = 0; e < VC / (4 / ES); ++e) {
                        x[e] = 0;
                        if (d + (4 / ES) * e < p.D) __builtin_memcpy(&x[e], p.cache.v + (at + d + (4 / ES) * e) * ES, 4);
                    }
                }
#pragma unroll
                for (int e = 0; e < VC / (4 / ES); ++e) v[u][i][e] = ok ? x[e] : 0u;
                if constexpr (CODES) {
                    ks[u][i] = p.cache.k_scale[scale];
                    vs[u][i] = ok ? p.cache.v_scale[scale] : 0.0f;
                }
            }
        }
        // ---- scores
        float x[2][4];
        float top = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            at_f4 acc{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                uint4 a;
                if constexpr (CODES)
                    a = make_uint4(codes2<T, false>(k[u][j][0]), codes2<T, true>(k[u][j][0]), codes2<T, false>(k[u][j][1]), codes2<T, true>(k[u][j][1]));
                else
                    a = make_uint4(k[u][j][0], k[u][j][1], k[u][j][2], k[u][j][3]);
                acc = mma<T>(a, q[j], acc);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y = acc[i] * p.scale;
                if constexpr (CODES) y *= ks[u][i];
                x[u][i] = live[u][i] ? y : -__builtin_inff();
                top = fmaxf(top, x[u][i]);
                seen |= live[u][i];
            }
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // (f16 probabilities are 2^15 times as large, so that small ones keep their bits: 2^-39 of the largest is the least)
        const float m_new = fmaxf(m, top), base = m_new == -__builtin_inff() ? 0.0f : m_new - (__is_same(VT, _Float16) ? 15.0f : 0.0f);
        const float alpha = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < VC; ++c) o[c] *= alpha;
        // ---- probabilities, each as the sum of two parts of VT, which together have twice its bits; the matrix core has time for it
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                float a = __builtin_amdgcn_exp2f(x[u][i] - base), b = __builtin_amdgcn_exp2f(x[u][i + 1] - base);
                l += a + b;
                if constexpr (CODES) {
                    a *= vs[u][i];
                    b *= vs[u][i + 1];
                }
                const uint32_t h = pack2<VT>(a, b);
                hi[2 * u + i / 2] = h;
                lo[2 * u + i / 2] = pack2<VT>(a - low_of<VT>(h), b - high_of<VT>(h));
            }
        const uint4 ph = make_uint4(hi[0], hi[1], hi[2], hi[3]), pl = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        // ---- V^T P^T: column VC n + c of the eight tokens
#pragma unroll
        for (int c = 0; c < VC; c += 2) {
            uint32_t even[4], odd[4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    uint32_t a, b;
                    if constexpr (CODES) {
                        a = c % 4 ? codes2<VT, true>(v[u][i][c / 4]) : codes2<VT, false>(v[u][i][c / 4]);
                        b = c % 4 ? codes2<VT, true>(v[u][i + 1][c / 4]) : codes2<VT, false>(v[u][i + 1][c / 4]);
                    } else {
                        a = v[u][i][c / 2];
                        b = v[u][i + 1][c / 2];
                    }
                    even[2 * u + i / 2] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                    odd[2 * u + i / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                }
            const uint4 ve = make_uint4(even[0], even[1], even[2], even[3]), vo = make_uint4(odd[0], odd[1], odd[2], odd[3]);
            o[c] = mma<VT>(ve, pl, mma<VT>(ve, ph, o[c]));
            o[c + 1] = mma<VT>(vo, pl, mma<VT>(vo, ph, o[c + 1]));
        }
    }

    // ---- the four groups of a head's tokens, then the waves
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) tops[wave][n] = m;
    const bool any = __syncthreads_or(seen);
    float top = tops[0][n];
#pragma unroll
    for (int w = 1; w < TK_WAVES; ++w) top = fmaxf(top, tops[w][n]);
    const float alpha = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    l *= alpha;
#pragma unroll
    for (int c = 0; c < VC; ++c) o[c] *= alpha;
    // lane: head n, columns VC (4 g + i) + c
#pragma unroll
    for (int half = TK_WAVES / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c) joined[wave - half][n][VC * (4 * g + i) + c] = o[c][i];
            if (g == 0) joined[wave - half][n][DP] = l;
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c) o[c][i] += joined[wave][n][VC * (4 * g + i) + c];
            l += joined[wave][n][DP];
        }
        __syncthreads();
    }
    if (wave != 0 || n >= cols) return;
    if (p.parts == 1) {
        // (a row whose every score is -inf has l = 0 and comes out as NaN, as its definition does; a row without tokens as 0)
        const float r = any ? 1.0f / l : 0.0f;
        T *to = static_cast<T *>(p.o) + s * p.ldo + (int64_t)(head0 + n) * p.D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < VC; c += 2) {
                const int d = VC * (4 * g + i) + c;
                const uint32_t w = any ? pack2<T>(o[c][i] * r, o[c + 1][i] * r) : 0u;
                if (FAST || d < p.D) __builtin_memcpy(to + d, &w, 4);
            }
    } else {
        float *to = p.partial + (((int64_t)s * p.Hq + head0 + n) * p.parts + blockIdx.x) * (p.D + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < VC; c += 2) {
                const int d = VC * (4 * g + i) + c;
                const f8_f2 w{o[c][i], o[c + 1][i]};
                if (FAST || d < p.D) __builtin_memcpy(to + d, &w, 8);
            }
        if (g == 0) {
            to[p.D] = top;
            to[p.D + 1] = any ? l : -1.0f;                               // (no token of the chunk was there)
        }
    }
}

// Joins the parts of a head: a workgroup for each sequence and query head, D / 4 lanes a part.
template <typename T>
__global__ void __launch_bounds__(256) k_attention_join(const TokenParams p)
{
    __shared__ float sums[256][5];
    const int s = blockIdx.y, h = blockIdx.x;
    const int length = min(max(__builtin_amdgcn_readfirstlane(p.length[s]), 0), p.max_length);
    const int chunk = chunk_of(p, length);
    const int parts = max(1, (length + chunk - 1) / chunk);
    const float *from = p.partial + ((int64_t)s * p.Hq + h) * p.parts * (p.D + 4);
    const int per = p.D / 4, at = threadIdx.x % per, lane0 = threadIdx.x / per, step = 256 / per;
    float m = -__builtin_inff();
    bool any = false;
    for (int i = 0; i < parts; ++i) {
        const float l = from[(int64_t)i * (p.D + 4) + p.D + 1];
        any |= !(l < 0.0f);
        if (!(l < 0.0f)) m = fmaxf(m, from[(int64_t)i * (p.D + 4) + p.D]);
    }
    at_f4 o{0, 0, 0, 0};
    float l = 0.0f;
    if (lane0 < step)
        for (int i = lane0; i < parts; i += step) {
            const float *x = from + (int64_t)i * (p.D + 4);
            const float mi = x[p.D], li = x[p.D + 1];
            if (li < 0.0f) continue;
            const float w = mi == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(mi - m);
            at_f4 y;
            __builtin_memcpy(&y, x + 4 * at, 16);
            o += y * w;
            l = fmaf(li, w, l);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[threadIdx.x][i] = o[i];
    sums[threadIdx.x][4] = l;
    __syncthreads();
    if (threadIdx.x >= per) return;
    for (int k = 1; k < step; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += sums[threadIdx.x + k * per][i];
        l += sums[threadIdx.x + k * per][4];
    }
    const float r = any ? 1.0f / l : 0.0f;
    const uint2 w = any ? make_uint2(pack2<T>(o[0] * r, o[1] * r), pack2<T>(o[2] * r, o[3] * r)) : make_uint2(0, 0);
    __builtin_memcpy(static_cast<T *>(p.o) + s * p.ldo + (int64_t)h * p.D + 4 * at, &w, 8);
}

// ---- host ------------------------------------------------------------------------------------------------------

// The most parts that a sequence is split into.  About two workgroups to a compute unit are wanted; where lengths differ, the longest get
// up to four times their even share.  A part has 128 tokens or more.
static int most_parts(int64_t sequences, int64_t blocks, int64_t max_length, int *target)
{
    *target = 512;
    if (sequences * blocks >= 2 * *target) return 1;
    const int64_t even = ceil_div(*target, sequences * blocks), slack = sequences > 1 ? 4 : 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(even * slack, max_length / (TK_WAVES * TK_TILE)));
}

static int64_t head_blocks(int q_heads, int kv_heads) { return kv_heads * ceil_div(q_heads / kv_heads, TK_COLS); }

template <typename T, bool CODES, int DP>
static void launch_token(const TokenParams &p, bool fast, hipStream_t s)
{
    const dim3 grid(p.parts, p.Hkv * p.col_tiles, p.sequences);
    if (fast && p.D == DP)
        k_attention_token<T, CODES, DP, true><<<grid, TK_WAVES * 64, 0, s>>>(p);
    else
        k_attention_token<T, CODES, DP, false><<<grid, TK_WAVES * 64, 0, s>>>(p);
}

template <typename T>
static nq_status run_token(const TokenParams &p, bool fast, hipStream_t s)
{
    auto by_dim = [&](auto codes) {
        constexpr bool C = decltype(codes)::value;
        if (p.D <= 64)
            launch_token<T, C, 64>(p, fast, s);
        else if (p.D <= 128)
            launch_token<T, C, 128>(p, fast, s);
        else
            launch_token<T, C, 256>(p, fast, s);
    };
    if (p.cache.type == NQ_KV_E4M3)
        by_dim(std::true_type{});
    else
        by_dim(std::false_type{});
    const nq_status st = launch_status();
    if (st != NQ_OK || p.parts == 1) return st;
    k_attention_join<T><<<dim3(p.Hq, p.sequences), 256, 0, s>>>(p);
    return launch_status();
}

}  // namespace nq

using namespace nq;

extern "C" size_t nq_attention_token_workspace_bytes(int64_t sequences, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_length)
{
    if (sequences < 1 || max_length < 1 || sequences > ATT_MAX_ROWS || max_length > INT32_MAX) return 0;
    if (check_heads(q_heads, kv_heads, head_dim) != NQ_OK || q_heads % kv_heads) return 0;
    int target;
    const int parts = most_parts(sequences, head_blocks(q_heads, kv_heads), max_length, &target);
    return parts == 1 ? 0 : (size_t)sequences * q_heads * parts * (head_dim + 4) * sizeof(float);
}

extern "C" nq_status nq_attention_token(const nq_token_job *job, void *stream)
{
    if (!job || job->sequences < 0 || job->max_length < 0 || job->ldtable < 0) return NQ_ERR_INVALID_ARG;
    const nq_token_job &j = *job;
    if (!is_dtype(j.dtype)) return NQ_ERR_INVALID_ARG;
    nq_status st = check_cache(j.cache);
    if (st != NQ_OK) return st;
    const nq_kv_cache &c = *j.cache;
    if ((st = check_heads(j.q_heads, c.heads, c.head_dim)) != NQ_OK) return st;
    if (j.q_heads % c.heads) return NQ_ERR_SHAPE;
    if (j.dtype == NQ_DT_F32 || (c.type != NQ_KV_E4M3 && c.type != j.dtype)) return NQ_ERR_UNSUPPORTED;
    if (j.sequences > 65535 || j.max_length > INT32_MAX - 4096 || j.ldtable > (int64_t(1) << 32)) return NQ_ERR_SHAPE;
    if (j.sequences == 0) return NQ_OK;
    const int64_t width = (int64_t)j.q_heads * c.head_dim;
    if ((st = check_matrix(j.d_q, j.dtype, width, j.ldq)) != NQ_OK) return st;
    if ((st = check_matrix(j.d_o, j.dtype, width, j.ldo)) != NQ_OK) return st;
    if (!j.d_length || (!j.d_table && j.max_length > 0)) return NQ_ERR_INVALID_ARG;
    if (!aligned_to(j.d_length, 4) || !aligned_to(j.d_table, 4)) return NQ_ERR_ALIGN;
    if (j.ldtable * c.page_tokens < j.max_length) return NQ_ERR_SHAPE;

    TokenParams p;
    p.q = j.d_q;
    p.o = j.d_o;
    p.table = j.d_table;
    p.length = j.d_length;
    p.partial = static_cast<float *>(j.d_workspace);
    p.cache = view_of(c);
    p.ldq = j.ldq;
    p.ldo = j.ldo;
    p.ldtable = j.ldtable;
    p.sequences = (int32_t)j.sequences;
    p.max_length = c.pages == 0 ? 0 : (int32_t)j.max_length;      // (a cache without pages has no token)
    p.Hq = j.q_heads;
    p.Hkv = c.heads;
    p.group = j.q_heads / c.heads;
    p.col_tiles = (int32_t)ceil_div(p.group, TK_COLS);
    p.D = c.head_dim;
    p.scale = j.scale * TK_LOG2E;
    p.parts = most_parts(p.sequences, head_blocks(j.q_heads, c.heads), j.max_length, &p.target);
    if (p.parts > 1) {
        if (!j.d_workspace) return NQ_ERR_INVALID_ARG;
        if (!aligned16(j.d_workspace)) return NQ_ERR_ALIGN;
        if (j.workspace_bytes < nq_attention_token_workspace_bytes(j.sequences, j.q_heads, c.heads, c.head_dim, j.max_length)) return NQ_ERR_RANGE;
    }
    const bool fast = c.page_tokens % 16 == 0;
    return j.dtype == NQ_DT_F16 ? run_token<_Float16>(p, fast, (hipStream_t)stream) : run_token<bf16_t>(p, fast, (hipStream_t)stream);
}
