// nq_attention_token: attention of one new token of each sequence over the paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(x_j - m),  x_j = scale log2(e) (q . k_j),  m the largest x so far
//
// Bound by the bytes of the cache's keys and values, each of which is read once (once for every 16 query heads of a group), straight into
// registers in the matrix instructions' operand order: S^T = K Q^T of 16 tokens x 32 columns x 16 query heads (those of one key head; a group of fewer leaves columns
// empty, which the matrix core has time for), then O^T = V^T P^T of 32 tokens.  The lane that holds four tokens' scores of a head
// after the first product holds the same tokens' place in the second one's operand, because the order in which a product sums its
// tokens is free: the probabilities never leave their registers, and a lane keeps the maximum and the sum of one head.
// 4 sequences of 65536 tokens, 8 key heads of 128 bf16: 189 us, 5.7 TB/s; 96 of 64 to 4096, e4m3, 56 us, 3.8 TB/s, the rest of it the pieces'
// uneven ends and the planning; one sequence of 517 tokens 9.6 us, a launch and the chain of five steps of one workgroup to a key head.
#include "nq_attention.h"

namespace nq {

typedef __bf16 at_b8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_h2 __attribute__((ext_vector_type(2)));
typedef float at_f4 __attribute__((ext_vector_type(4)));

constexpr int TK_TILE = 32, TK_COLS = 16;                  // tokens of a wave's step; query heads of a matrix tile
constexpr float TK_LOG2E = 1.44269504088896340736f;

constexpr int TK_LEAST = 128, TK_MOST_PLANNED = 1024;      // tokens of a piece, at least; sequences of a call that is split, at most
// Workgroups to a compute unit, by their registers.
__host__ __device__ constexpr int workgroups_of(int head_dim, bool codes) { return head_dim <= 128 ? 3 : codes ? 2 : 1; }

struct TokenParams {
    const void *q;
    void *o;
    const int32_t *table, *length;
    float *partial;                       // sums of o [pieces][q_heads][D], then m and l [pieces][q_heads][2]
    int2 *dealt;                          // for each sequence: its first piece, how many it has
    CacheView cache;
    int64_t ldq, ldo, ldtable;
    int32_t sequences, max_length, Hq, Hkv, group, col_tiles, D, pieces;   // pieces: 0 where no sequence is split
    float share;                          // of all tokens, for a workgroup
    float scale;                          // times log2(e)
};

// How the call's tokens are dealt to workgroups.  chunk is the share of each if all tokens were dealt evenly to as many as the card holds.  A sequence
// of more than half a chunk goes into pieces of equal size, as few as have a chunk at most; those come first, and the shorter sequences,
// a piece each, fill the gaps that they leave.  So there are as many pieces as workgroups wanted, and one more for each sequence, at most.
// Every wave that asks makes the same sums in the same order.
__device__ __forceinline__ int length_of(const TokenParams &p, int i) { return i < p.sequences ? min(max(p.length[i], 0), p.max_length) : 0; }

// The call's lengths, a lane each of 64 sequences, 256 asked for at once and kept if there are no more.
struct Lengths {
    const TokenParams &p;
    int at, held[4];
    __device__ __forceinline__ explicit Lengths(const TokenParams &params) : p(params) { ask(0); }
    __device__ __forceinline__ void ask(int from)
    {
        at = from;
#pragma unroll
        for (int r = 0; r < 4; ++r) held[r] = length_of(p, from + 64 * r + (threadIdx.x & 63));
    }
    // f(first of 64 sequences, this lane's length), until it returns true
    template <typename F>
    __device__ __forceinline__ void each(F f)
    {
        for (int i = 0; i < p.sequences; i += 256) {
            if (at != i) ask(i);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (i + 64 * r < p.sequences && f(i + 64 * r, held[r])) return;
        }
    }
};

__device__ __forceinline__ int chunk_of(const TokenParams &p, Lengths &lengths)
{
    float total = 0.0f;
    lengths.each([&](int, int length) {
        total += (float)length;
        return false;
    });
    const float even = fminf(ceilf(sum64(total) * p.share), 2147483520.0f);
    return __builtin_amdgcn_readfirstlane((max((int)even, TK_LEAST) + TK_TILE - 1) / TK_TILE * TK_TILE);
}
struct Pieces {
    int first, count, size;               // numbers of a sequence's pieces, tokens of one
};
// Calls found(sequence, length, Pieces) for 64 sequences at a time, a lane each, until it says that that was it.
template <typename F>
__device__ __forceinline__ void each_sequence(const TokenParams &p, F found)
{
    const int lane = threadIdx.x & 63;
    Lengths lengths(p);
    const int chunk = chunk_of(p, lengths);
    auto pieces = [&](int length) {
        const int n = max((int)(((uint32_t)length + (uint32_t)chunk - 1) / (uint32_t)chunk), 1), size = max(((length + n - 1) / n + TK_TILE - 1) / TK_TILE * TK_TILE, TK_TILE);
        return Pieces{0, max((length + size - 1) / size, 1), size};
    };
    auto large = [&](int length) { return length > chunk / 2; };
    int behind = 0, first = 0, all;                                      // behind: pieces of the large sequences
    if (p.sequences > 64) {
        lengths.each([&](int, int length) {
            behind += large(length) ? pieces(length).count : 0;
            return false;
        });
        (void)before(behind, &behind);
    }
    lengths.each([&](int i, int length) {
        const bool is = large(length);
        Pieces x = pieces(length);
        const int here = before(is ? x.count : 0, &all);
        if (p.sequences <= 64) behind = all;
        const uint64_t mask = __ballot(!is && i + lane < p.sequences);
        x.first = is ? first + here : behind + __popcll(mask & ((uint64_t(1) << lane) - 1));
        if (i + lane >= p.sequences) x.count = 0;
        first += all;
        behind += __popcll(mask);
        return found(i + lane, length, x);
    });
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

// What a lane holds of 32 tokens, half u of them 16.  k: token n of a half, columns 32 j + 8 g; v: tokens 4 g + i, columns column(n, c).
template <int KJ, int KW, int VW>
struct TokenTile {
    uint32_t k[2][KJ][KW], v[2][4][VW];
    float scale;                          // of token n of half (lane / 32): its key's (lanes 0 .. 15 of the half wave) or its value's
    uint32_t live;                        // bit 4 u + i: token 4 g + i of half u is there
};

// T: queries and outputs; CODES: an e4m3 cache; DP: columns, head_dim rounded up to a form; CUT: head_dim < DP.
template <typename T, bool CODES, int DP, bool CUT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : workgroups_of(DP, CODES)) k_attention_token(const TokenParams p)
{
    constexpr int KJ = DP / 32, VC = DP / 16, RUN = VC < 8 ? VC : 8, ES = CODES ? 1 : 2;      // products to a score; columns of V to a lane, and beside each other
    constexpr int KW = CODES ? 2 : 4, VW = VC / (4 / ES), RW = RUN / (4 / ES);                // dwords of eight elements; of VC; of RUN
    constexpr int STEP = WAVES * TK_TILE;
    using VT = typename std::conditional<CODES, bf16_t, T>::type;       // codes times their scale: bf16's range, in two parts
    using Tile = TokenTile<KJ, KW, VW>;
    __shared__ __attribute__((aligned(16))) float joined[WAVES / 2][TK_COLS][DP + 4];
    __shared__ float tops[WAVES][TK_COLS];
    __shared__ __attribute__((aligned(16))) float scales[WAVES][64];
    __shared__ __attribute__((aligned(16))) int64_t rows[WAVES][TK_TILE];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    // (heads first: neighbouring workgroups go to the eight dies in turn)
    const int hk = blockIdx.x / p.col_tiles, col0 = (blockIdx.x - hk * p.col_tiles) * TK_COLS, piece = blockIdx.y;
    const int cols = min(TK_COLS, p.group - col0), head0 = hk * p.group + col0;
    int s = piece, begin = 0, end = 0;
    bool whole = true;
    if (p.pieces) {
        s = -1;
        each_sequence(p, [&](int i, int length, const Pieces &x) {
            const uint64_t mask = __ballot(piece >= x.first && piece < x.first + x.count);
            if (!mask) return false;
            const int from = __builtin_ctzll(mask), at = (piece - x.first) * x.size;
            s = __builtin_amdgcn_readlane(i, from);
            begin = __builtin_amdgcn_readlane(at, from);
            end = __builtin_amdgcn_readlane(at + min(length - at, x.size), from);
            const int count = __builtin_amdgcn_readlane(x.count, from), first_piece = __builtin_amdgcn_readlane(x.first, from);
            whole = count == 1;
            // (for the join; every sequence has a first piece)
            if (blockIdx.x == 0 && piece == first_piece && threadIdx.x == 0) p.dealt[s] = make_int2(first_piece, count);
            return true;
        });
        if (s < 0) return;
    } else {
        end = __builtin_amdgcn_readfirstlane(length_of(p, s));
    }
    auto column = [&](int c) { return RUN * n + (c / RUN) * 16 * RUN + c % RUN; };

    // ---- loading, in three steps: the page of a token, where its row is, the row
    const int32_t *table = p.table + s * p.ldtable;
    const int mine = 16 * (lane >> 5) + n;                              // the token of 32 that this lane looks up
    auto token_at = [&](int t0) { return (uint32_t)min(t0 + mine, end - 1); };
    auto page_of = [&](int t0) { return table[divide(token_at(t0), p.cache.by_page)]; };
    const uint8_t *k_head = p.cache.k + hk * p.cache.head_step * ES, *v_head = p.cache.v + hk * p.cache.head_step * ES;
    const float *scale_head = (lane & 16 ? p.cache.v_scale : p.cache.k_scale) + hk * p.cache.scale_head_step;
    auto load = [&](Tile &x, int t0, int32_t page) {
        const uint32_t t = token_at(t0), place = t - divide(t, p.cache.by_page) * p.cache.by_page.d;
        const bool there = t0 + mine < end && (uint32_t)page < (uint32_t)p.cache.pages;
        const int64_t row = (int64_t)page * p.cache.page_step + (int64_t)place * p.cache.token_step;
        rows[wave][mine] = there ? row : -1;                             // (two lanes write the same)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();                                 // (LDS serves a wave's requests in order)
        if constexpr (CODES) x.scale = scale_head[there ? (int64_t)page * p.cache.scale_page_step + (int64_t)place * p.cache.scale_token_step : 0];
        x.live = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // (a token that is not there: the cache's first, whose value is not used)
            const uint8_t *k = k_head + max(rows[wave][16 * u + n], (int64_t)0) * ES;
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                const int d = 32 * j + 8 * g;
                __builtin_memcpy(x.k[u][j], k + (CUT && d >= p.D ? 0 : d) * ES, sizeof x.k[u][j]);
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t at = rows[wave][16 * u + 4 * g + i];
                x.live |= at >= 0 ? 1u << (4 * u + i) : 0u;
                const uint8_t *v = v_head + max(at, (int64_t)0) * ES;
#pragma unroll
                for (int c = 0; c < VC; c += RUN)
                    __builtin_memcpy(&x.v[u][i][c / RUN * RW], v + (CUT && column(c) >= p.D ? 0 : column(c)) * ES, RW * 4);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    uint4 q[KJ];
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
        q[j] = make_uint4(0, 0, 0, 0);
        const int d = 32 * j + 8 * g;
        if (n < cols && (!CUT || d < p.D)) __builtin_memcpy(&q[j], static_cast<const T *>(p.q) + s * p.ldq + (int64_t)(head0 + n) * p.D + d, 16);
    }

    at_f4 o[VC];
#pragma unroll
    for (int c = 0; c < VC; ++c) o[c] = at_f4{0, 0, 0, 0};
    float m = -__builtin_inff(), l = 0.0f;
    bool seen = false;

    auto attend = [&](Tile &y) {
        float ks[2][4], vs[2][4];
        if constexpr (CODES) {                                          // (LDS serves a wave's requests in order)
            scales[wave][lane] = y.scale;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        // ---- scores
        float x[2][4];
        at_f4 acc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            acc[u] = at_f4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                if (CUT && 32 * j + 8 * g >= p.D) {
#pragma unroll
                    for (int i = 0; i < KW; ++i) y.k[u][j][i] = 0;
                }
                uint4 a;
                if constexpr (CODES)
                    a = make_uint4(codes2<T, false>(y.k[u][j][0]), codes2<T, true>(y.k[u][j][0]), codes2<T, false>(y.k[u][j][1]), codes2<T, true>(y.k[u][j][1]));
                else
                    a = make_uint4(y.k[u][j][0], y.k[u][j][1], y.k[u][j][2], y.k[u][j][3]);
                acc[u] = mma<T>(a, q[j], acc[u]);
            }
        }
        if constexpr (CODES) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                __builtin_memcpy(ks[u], &scales[wave][32 * u + 4 * g], 16);
                __builtin_memcpy(vs[u], &scales[wave][32 * u + 16 + 4 * g], 16);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[u][i] = acc[u][i] * p.scale;
                if constexpr (CODES) x[u][i] *= ks[u][i];
            }
        if (!__all(y.live == 0xffu)) {
            // what is not there has no weight, and no value that could be infinite or NaN
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(y.live >> (4 * u + i) & 1)) {
                        x[u][i] = -__builtin_inff();
                        if constexpr (CODES) vs[u][i] = 0.0f;
#pragma unroll
                        for (int e = 0; e < VW; ++e) y.v[u][i][e] = 0;
                    }
            seen |= y.live != 0;
        } else {
            seen = true;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, x[u][i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // (f16 probabilities are 2^15 times as large, so that small ones keep their bits: 2^-39 of the largest is the least)
        const float m_new = fmaxf(m, top), base = m_new == -__builtin_inff() ? 0.0f : m_new - (__is_same(VT, _Float16) ? 15.0f : 0.0f);
        if (__any(m_new > m)) {                                         // (seldom after the first tokens)
            const float alpha = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < VC; ++c) o[c] *= alpha;
        }
        // ---- probabilities, each as the sum of two parts of VT, which together have twice its bits (off by 2^-17 of it for bf16, 2^-23 for f16); the
        // matrix core has time for it
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
                        a = c % 4 ? codes2<VT, true>(y.v[u][i][c / 4]) : codes2<VT, false>(y.v[u][i][c / 4]);
                        b = c % 4 ? codes2<VT, true>(y.v[u][i + 1][c / 4]) : codes2<VT, false>(y.v[u][i + 1][c / 4]);
                    } else {
                        a = y.v[u][i][c / 2];
                        b = y.v[u][i + 1][c / 2];
                    }
                    even[2 * u + i / 2] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                    odd[2 * u + i / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                }
            const uint4 ve = make_uint4(even[0], even[1], even[2], even[3]), vo = make_uint4(odd[0], odd[1], odd[2], odd[3]);
            o[c] = mma<VT>(ve, pl, mma<VT>(ve, ph, o[c]));
            o[c + 1] = mma<VT>(vo, pl, mma<VT>(vo, ph, o[c + 1]));
        }
    };

    int t0 = begin + wave * TK_TILE;
    if (t0 < end) {
        // The pages of the next tokens are looked up ahead (behind the last ones, theirs again).  The next tokens themselves are not: three
        // workgroups to a compute unit cover the memory's latency as well as twice the registers do (4 x 65536 tokens of bf16 187 us, with
        // two tiles in registers 186; 256 x 1024 of e4m3 51.6 and 55.5).
        auto next = [&](int t) { return t + STEP < end ? t + STEP : t; };
        Tile x;
        int32_t page = page_of(t0), after = page_of(next(t0));
        for (;;) {
            load(x, t0, page);
            page = after;
            after = page_of(next(next(t0)));
            attend(x);
            if ((t0 += STEP) >= end) break;
        }
    }

    // ---- the four groups of a head's tokens, then the waves
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) tops[wave][n] = m;
    const bool any = __syncthreads_or(seen);
    float top = tops[0][n];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w][n]);
    const float alpha = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    l *= alpha;
#pragma unroll
    for (int c = 0; c < VC; ++c) o[c] *= alpha;
    // lane: head n, columns of the rows 4 g + i of the product
    auto column_of = [&](int i, int c) { return RUN * (4 * g + i) + (c / RUN) * 16 * RUN + c % RUN; };
#pragma unroll
    for (int half = WAVES / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c) joined[wave - half][n][column_of(i, c)] = o[c][i];
            if (g == 0) joined[wave - half][n][DP] = l;
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < VC; ++c) o[c][i] += joined[wave][n][column_of(i, c)];
            l += joined[wave][n][DP];
        }
        __syncthreads();
    }
    if (wave != 0 || n >= cols) return;
    if (whole) {
        // (a row whose every score is -inf has l = 0 and comes out as NaN, as its definition does; a row without tokens as 0)
        const float r = any ? 1.0f / l : 0.0f;
        T *to = static_cast<T *>(p.o) + s * p.ldo + (int64_t)(head0 + n) * p.D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < VC; c += 2) {
                const int d = column_of(i, c);
                const uint32_t w = any ? pack2<T>(o[c][i] * r, o[c + 1][i] * r) : 0u;
                if (!CUT || d < p.D) __builtin_memcpy(to + d, &w, 4);
            }
    } else {
        const int64_t row = (int64_t)piece * p.Hq + head0 + n;
        float *to = p.partial + row * p.D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < VC; c += 2) {
                const int d = column_of(i, c);
                const f8_f2 w{o[c][i], o[c + 1][i]};
                if (!CUT || d < p.D) __builtin_memcpy(to + d, &w, 8);
            }
        if (g == 0)                                                      // (a sum of -1: no token of the piece was there)
            reinterpret_cast<f8_f2 *>(p.partial + (int64_t)p.pieces * p.Hq * p.D)[row] = f8_f2{top, any ? l : -1.0f};
    }
}

// Joins the pieces of a sequence: TH threads for each query head.  All loads are on their way at once: a thread asks for the
// maximum and sum of one piece, and for four columns of every (4 TH / D)-th.
template <typename T, int TH>
__global__ void __launch_bounds__(256) k_attention_join(const TokenParams p)
{
    constexpr int AHEAD = TH == 64 ? 8 : 4, HEADS = 256 / TH;
    __shared__ float sums[HEADS][TH][5], weight[HEADS][TH], tops[4];
    const int s = blockIdx.y, group = threadIdx.x / TH, tid = threadIdx.x % TH, h = min((int)blockIdx.x * HEADS + group, p.Hq - 1);
    const int2 dealt = p.dealt[s];
    const Pieces all{dealt.x, dealt.y, 0};
    if (all.count <= 1) return;                                          // (k_attention_token has written the row)
    const f8_f2 *ml = reinterpret_cast<const f8_f2 *>(p.partial + (int64_t)p.pieces * p.Hq * p.D);
    const int per = p.D / 4, at = tid % per, mine = tid / per, step = TH / per;
    auto row = [&](int i) { return (int64_t)(all.first + i) * p.Hq + h; };
    float m = -__builtin_inff(), l = 0.0f;
    bool any = false;
    at_f4 o{0, 0, 0, 0};
    for (int base = 0; base < all.count; base += TH) {
        const int count = min(all.count - base, TH);
        f8_f2 x{-__builtin_inff(), -1.0f};
        if (tid < count) x = ml[row(base + tid)];
        at_f4 y[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (mine < step && mine + i * step < count) __builtin_memcpy(&y[i], p.partial + row(base + mine + i * step) * p.D + 4 * at, 16);
        const bool there = !(x[1] < 0.0f);                               // (a piece without any token has no weight)
        float top = there ? x[0] : -__builtin_inff();
#pragma unroll
        for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
        if (TH > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        }
        any |= __syncthreads_or(there) != 0;                             // (the same tokens for every head of the sequence)
        if (TH > 64) top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        const float m_new = fmaxf(top, m);
        const float keep = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - m_new);
        const float w = !there || x[0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(x[0] - m_new);
        m = m_new;
        weight[group][tid] = w;
        l = l * keep + (there ? x[1] * w : 0.0f);
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] *= keep;
        // (a piece without weight counts, too: 0 times an infinite or NaN value is no 0; a piece without any token holds zeros)
        auto add = [&](int i, const at_f4 &z) {
            const float v = weight[group][i];
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(z[c], v, o[c]);
        };
        if (mine < step) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (mine + i * step < count) add(mine + i * step, y[i]);
            for (int i = mine + AHEAD * step; i < count; i += step) {
                at_f4 z;
                __builtin_memcpy(&z, p.partial + row(base + i) * p.D + 4 * at, 16);
                add(i, z);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[group][tid][i] = o[i];
    sums[group][tid][4] = l;
    __syncthreads();
    if (tid >= per || (int)blockIdx.x * HEADS + group >= p.Hq) return;
    for (int k = 1; k < step; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += sums[group][tid + k * per][i];
    l = 0.0f;
    for (int k = 0; k < min(TH, all.count); ++k) l += sums[group][k][4];
    const float r = any ? 1.0f / l : 0.0f;
    const uint2 w = any ? make_uint2(pack2<T>(o[0] * r, o[1] * r), pack2<T>(o[2] * r, o[3] * r)) : make_uint2(0, 0);
    __builtin_memcpy(static_cast<T *>(p.o) + s * p.ldo + (int64_t)h * p.D + 4 * at, &w, 8);
}

// ---- host ------------------------------------------------------------------------------------------------------

// Calls of short sequences that do not fill the card: eight waves to a workgroup and no pieces to join, a second launch saved (one sequence of
// 517 tokens 9.6 us, in pieces 10.5; of 1000 tokens 13.7 and 10.5; of 100, which four waves take in one step, 5.9 and 5.5).
static bool short_call(int64_t sequences, int64_t blocks, int64_t max_length, int head_dim)
{
    return head_dim <= 128 && max_length > TK_LEAST && max_length <= 640 && sequences * blocks <= 256;
}

// Pieces of the call's tokens for each of `blocks` head blocks, 0: a sequence is one.  `target` workgroups are wanted.  Two to a compute unit carry the
// memory's rate and leave the third's place to what is short (64 sequences of 1024 tokens, 128 columns e4m3, 32.4 us, for three 37.6; 64 columns bf16,
// whose tiles are smaller, 42.6 and 39.8).  From twice that many sequences on they even out by themselves, unless one may be so long that its
// workgroup is the last for a while; against that stands the planning, which each workgroup does over all sequences.  8 key heads of 128 e4m3, whole
// and in pieces: 256 sequences of up to 1024 tokens 40.7 and 43.6 us, to 2048 72.5 and 67.1, one of 65536 among 255 of some 200 609 and 59;
// 512 of up to 4096 235 and 265, one of 32768 among short ones 354 and 95; one of 16384 among 999 232 and 220.
static int64_t pieces_of(int64_t sequences, int64_t blocks, int64_t max_length, int head_dim, int64_t *target)
{
    *target = 256 * (head_dim <= 64 ? 3 : 2);
    if (max_length <= TK_LEAST || sequences > TK_MOST_PLANNED) return 0;
    if (sequences * blocks >= 2 * *target && (max_length < 2048 || sequences * sequences * blocks > 256 * max_length)) return 0;
    if (short_call(sequences, blocks, max_length, head_dim)) return 0;
    return std::min(ceil_div(*target, blocks) + 1, sequences * (max_length / TK_LEAST)) + sequences;
}

static int64_t head_blocks(int q_heads, int kv_heads) { return kv_heads * ceil_div(q_heads / kv_heads, TK_COLS); }

template <typename T, bool CODES, int DP, int WAVES>
static void launch_waves(const TokenParams &p, hipStream_t s)
{
    const dim3 grid(p.Hkv * p.col_tiles, p.pieces ? p.pieces : p.sequences);
    if (p.D == DP)
        k_attention_token<T, CODES, DP, false, WAVES><<<grid, WAVES * 64, 0, s>>>(p);
    else
        k_attention_token<T, CODES, DP, true, WAVES><<<grid, WAVES * 64, 0, s>>>(p);
}

template <typename T, bool CODES, int DP>
static void launch_token(const TokenParams &p, hipStream_t s)
{
    if constexpr (DP <= 128) {
        if (short_call(p.sequences, p.Hkv * p.col_tiles, p.max_length, DP)) return launch_waves<T, CODES, DP, 8>(p, s);
    }
    launch_waves<T, CODES, DP, 4>(p, s);
}

template <typename T>
static nq_status run_token(const TokenParams &p, hipStream_t s)
{
    auto by_dim = [&](auto codes) {
        constexpr bool C = decltype(codes)::value;
        if (p.D <= 64)
            launch_token<T, C, 64>(p, s);
        else if (p.D <= 128)
            launch_token<T, C, 128>(p, s);
        else
            launch_token<T, C, 256>(p, s);
    };
    if (p.cache.type == NQ_KV_E4M3)
        by_dim(std::true_type{});
    else
        by_dim(std::false_type{});
    const nq_status st = launch_status();
    if (st != NQ_OK || !p.pieces) return st;
    // a wave for a head, four where there are few heads and many pieces of them
    if (p.pieces - p.sequences <= 8 || p.sequences * p.Hq >= 1024)
        k_attention_join<T, 64><<<dim3((unsigned)ceil_div(p.Hq, 4), p.sequences), 256, 0, s>>>(p);
    else
        k_attention_join<T, 256><<<dim3(p.Hq, p.sequences), 256, 0, s>>>(p);
    return launch_status();
}

}  // namespace nq

using namespace nq;

extern "C" size_t nq_attention_token_workspace_bytes(int64_t sequences, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_length)
{
    if (sequences < 1 || max_length < 1 || sequences > ATT_MAX_ROWS || max_length > INT32_MAX) return 0;
    if (check_heads(q_heads, kv_heads, head_dim) != NQ_OK || q_heads % kv_heads) return 0;
    int64_t target;
    const int64_t blocks = head_blocks(q_heads, kv_heads);
    const int64_t pieces = pieces_of(sequences, blocks, max_length, head_dim, &target);
    return pieces ? (size_t)pieces * q_heads * (head_dim + 2) * sizeof(float) + (size_t)sequences * sizeof(int2) : 0;
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
    int64_t target;
    const int64_t blocks = head_blocks(j.q_heads, c.heads);
    p.pieces = (int32_t)pieces_of(p.sequences, blocks, j.max_length, c.head_dim, &target);
    p.dealt = reinterpret_cast<int2 *>(p.partial + (int64_t)p.pieces * p.Hq * (p.D + 2));
    p.share = (float)blocks / (float)target;
    if (p.pieces) {
        if (!j.d_workspace) return NQ_ERR_INVALID_ARG;
        if (!aligned16(j.d_workspace)) return NQ_ERR_ALIGN;
        if (j.workspace_bytes < nq_attention_token_workspace_bytes(j.sequences, j.q_heads, c.heads, c.head_dim, j.max_length)) return NQ_ERR_RANGE;
    }
    return j.dtype == NQ_DT_F16 ? run_token<_Float16>(p, (hipStream_t)stream) : run_token<bf16_t>(p, (hipStream_t)stream);
}
