// nq_head_norm: norms of the queries' and keys' heads, position rotation, keys and values into a paged cache; nq_cache_read: rows of
// the cache back.  Both are bound by the bytes: each value is read once, goes through registers, and is written once.
#include "nq_attention.h"

namespace nq {

struct HeadParams {
    const void *q, *k, *v;
    void *q_out, *k_out;
    int64_t ldq, ldk, ldv, ldq_out, ldk_out;
    const float *q_w, *q_b, *k_w, *k_b, *freq;
    const int32_t *position;
    const int64_t *slot;
    CacheView cache;
    int64_t T, first, last;                // rows of the call; of this launch
    float q_eps, k_eps, inv_D;
    int32_t Hq, Hk, Hv;                    // (0 for what is not there)
    int32_t q_kind, k_kind, D, rotary, pairs, cached, split;
};

// Sums and maxima over the LPH neighbouring lanes that hold a head.
template <int LPH>
__device__ __forceinline__ float sum_lanes(float v)
{
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    if (LPH >= 16) v += dpp<0x140>(v);
    if (LPH >= 32) v += __shfl_xor(v, 16);
    return v;
}
template <int LPH>
__device__ __forceinline__ uint32_t max_lanes(uint32_t v)
{
    v = max(v, dpp<0xB1>(v));
    v = max(v, dpp<0x4E>(v));
    v = max(v, dpp<0x141>(v));
    if (LPH >= 16) v = max(v, dpp<0x140>(v));
    if (LPH >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    return v;
}

// (cos, sin) of position * freq.  The angle in turns and its nearest quarter in 64 bits: a position of a million keeps 2^-32 of a
// turn, where fp32 has 2^-4 left.  What remains is within an eighth of a turn, where the Taylor series to x^9 and x^10 are good to
// 2e-9 and so to fp32's rounding.
__device__ __forceinline__ float2 turn_of(int32_t position, float freq)
{
    const double turns = (double)position * ((double)freq * 0.15915494309189533577);
    const double r = turns - rint(turns), quarter = rint(4.0 * r);
    const float x = (float)((r - 0.25 * quarter) * 6.28318530717958647693), y = x * x;
    float s = fmaf(y, 2.75573192e-6f, -1.98412698e-4f), c = fmaf(y, -2.75573192e-7f, 2.48015873e-5f);
    s = fmaf(y, s, 8.33333333e-3f);
    s = fmaf(y, s, -0.166666667f);
    s = fmaf(x * y, s, x);
    c = fmaf(y, c, -1.38888889e-3f);
    c = fmaf(y, c, 4.16666667e-2f);
    c = fmaf(y, c, -0.5f);
    c = fmaf(y, c, 1.0f);
    const int n = (int)quarter & 3;
    const float cs = n & 1 ? s : c, sn = n & 1 ? c : s;
    return make_float2(n == 1 || n == 2 ? -cs : cs, n >= 2 ? -sn : sn);
}

template <typename T>
__device__ __forceinline__ void put8(void *base, int64_t at, const float (&v)[8])
{
    store8(static_cast<T *>(base) + at, 8, v);
}

// Eight values that a lane holds of a head, and what it needs to turn them.
struct Turn {
    float cos[8], sin[8];                 // NEIGHBOURS: of the lane's four pairs; HALVES: of the pairs of its eight columns, the sine with its sign
};

// Norm over the head's values, which lie in LPH lanes.
template <int LPH>
__device__ __forceinline__ void norm8(float (&v)[8], int kind, const float (&w)[8], const float *b, float eps, float inv_D, int c, bool in)
{
    if (kind == NQ_NORM_NONE) return;
    float sum = 0.0f;
    if (kind == NQ_NORM_LAYER) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
        const float mean = sum_lanes<LPH>(sum) * inv_D;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = in ? v[e] - mean : 0.0f;
        sum = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
    const float r = inverse_root(sum_lanes<LPH>(sum) * inv_D + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * r * w[e];
    if (b && in) {
        float x[8];
        __builtin_memcpy(x, b + c, sizeof x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
}

// The value of the lane half a head on.
template <int LPH>
__device__ __forceinline__ float half_on(float v)
{
    if (LPH == 8) return dpp<0x1B>(dpp<0x141>(v));                   // mirrored in eight, then in four
    return dpp<0x128>(v);                                            // eight on in sixteen
}

// A wave takes a token, or every p.split-th few of its heads: LPH lanes of eight values a head, AHEAD steps asked for at once.  The angles
// are made once for all of the wave's heads, a pair or two to a lane; a lane then keeps those of its columns.  MODE: how the pairs lie: 0 none,
// 1 neighbours, 2 halves in whole eights (a lane's partner is another lane's eight), 3 halves anywhere, 4 halves of LPH lanes.
// A step takes heads of one kind, so that what depends on the kind is scalar.
template <typename T, int LPH, int MODE>
__global__ void __launch_bounds__(256) k_head_norm(const HeadParams p)
{
    constexpr int PER = 64 / LPH, AHEAD = sizeof(T) == 4 ? 2 : 4;
    __shared__ __attribute__((aligned(16))) float2 turns[4][NQ_HEAD_MAX_DIM / 2];
    __shared__ __attribute__((aligned(16))) float stage[4][64 * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = lane / LPH, c = (lane % LPH) * 8;
    const int half = p.rotary >> 1, q_steps = (p.Hq + PER - 1) / PER, k_steps = q_steps + (p.Hk + PER - 1) / PER, steps = k_steps + (p.Hv + PER - 1) / PER;
    const bool in = c < p.D;
    float *mine = stage[wave] + group * LPH * 8;                     // this head's values
    const int64_t item = (int64_t)blockIdx.x * 4 + wave, t = p.first + item / p.split;
    const int part = (int)(item % p.split);
    if (t >= p.last) return;
    auto settle = [] {                                               // (LDS serves a wave's requests in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    Raw8<T> raw[AHEAD];
    const T *q_row = static_cast<const T *>(p.q) + t * p.ldq, *k_row = static_cast<const T *>(p.k) + t * p.ldk, *v_row = static_cast<const T *>(p.v) + t * p.ldv;
    auto ask = [&](int from) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int step = from + a * p.split;
            const T *row = step < q_steps ? q_row : step < k_steps ? k_row : v_row;
            const int i = (step < q_steps ? step : step < k_steps ? step - q_steps : step - k_steps) * PER + group;
            raw[a] = Raw8<T>{};
            if (in && step < steps && i < (step < q_steps ? p.Hq : step < k_steps ? p.Hk : p.Hv)) __builtin_memcpy(&raw[a], row + i * p.D + c, sizeof raw[a]);
        }
    };
    int step = part;
    ask(step);
    float wq[8], wk[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.0f;
    if (p.q_w && in) __builtin_memcpy(wq, p.q_w + c, sizeof wq);
    if (p.k_w && in) __builtin_memcpy(wk, p.k_w + c, sizeof wk);

    int64_t slot = p.cached ? p.slot[t] : -1, at = 0, scale_at = 0;
    if (slot >= p.cache.slots) slot = -1;
    if (slot >= 0) {
        const Place l = place_of(p.cache, slot);
        at = l.page * p.cache.page_step + l.token * p.cache.token_step;
        scale_at = l.page * p.cache.scale_page_step + l.token * p.cache.scale_token_step;
    }
    Turn turn;
    const float2 *angle = turns[wave];
    if constexpr (MODE != 0) {
        const int32_t position = p.position[t];
        for (int i = lane; i < half; i += 64) turns[wave][i] = turn_of(position, p.freq[i]);
        settle();
        if constexpr (MODE == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 u = c + 2 * e < p.rotary ? angle[(c >> 1) + e] : make_float2(1.0f, 0.0f);
                turn.cos[e] = u.x;
                turn.sin[e] = u.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int d = c + e;
                const float2 u = d < p.rotary ? angle[d < half ? d : d - half] : make_float2(1.0f, 0.0f);
                turn.cos[e] = u.x;
                turn.sin[e] = d < half ? -u.y : u.y;
            }
        }
    }
    const int partner = c < half ? c + half : c < p.rotary ? c - half : c;

    for (; step < steps; step += AHEAD * p.split) {
        Raw8<T> now[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) now[a] = raw[a];
        ask(step + AHEAD * p.split);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int here = step + a * p.split;
            if (here >= steps) break;
            const int which = here < q_steps ? 0 : here < k_steps ? 1 : 2, i = (which == 0 ? here : which == 1 ? here - q_steps : here - k_steps) * PER + group;
            const bool there = in && i < (which == 0 ? p.Hq : which == 1 ? p.Hk : p.Hv);
            float v[8];
            raw_to_float(now[a], v);
            if (which < 2) {
                if (which == 0)
                    norm8<LPH>(v, p.q_kind, wq, p.q_b, p.q_eps, p.inv_D, c, in);
                else
                    norm8<LPH>(v, p.k_kind, wk, p.k_b, p.k_eps, p.inv_D, c, in);
                if constexpr (MODE == 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (c + 2 * e >= p.rotary) break;
                        const float x = v[2 * e], y = v[2 * e + 1];
                        v[2 * e] = fmaf(x, turn.cos[e], -(y * turn.sin[e]));
                        v[2 * e + 1] = fmaf(y, turn.cos[e], x * turn.sin[e]);
                    }
                } else if constexpr (MODE == 4) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = half_on<LPH>(v[e]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], turn.cos[e], y[e] * turn.sin[e]);
                } else if constexpr (MODE == 2) {
                    float y[8];
                    __builtin_memcpy(mine + c, v, sizeof v);
                    settle();
                    __builtin_memcpy(y, __builtin_assume_aligned(mine + partner, 16), sizeof y);
                    settle();
                    if (c < p.rotary) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], turn.cos[e], y[e] * turn.sin[e]);
                    }
                } else if constexpr (MODE == 3) {
                    __builtin_memcpy(mine + c, v, sizeof v);
                    settle();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int d = c + e;
                        const float y = mine[d < half ? d + half : max(d - half, 0)];
                        if (d < p.rotary) v[e] = fmaf(v[e], turn.cos[e], y * turn.sin[e]);
                    }
                    settle();
                }
                if (which == 0) {
                    if (there) put8<T>(p.q_out, t * p.ldq_out + i * p.D + c, v);
                    continue;
                }
                if (p.k_out && there) put8<T>(p.k_out, t * p.ldk_out + i * p.D + c, v);
            }
            if (slot < 0) continue;
            uint8_t *cache = which == 1 ? p.cache.k : p.cache.v;
            const int64_t to = at + i * p.cache.head_step + c;
            if (p.cache.type == NQ_KV_E4M3) {
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, abs_bits(v[e]));
                if (!in) m = 0;
                float inverse;
                const float s = fp8_scale(max_lanes<LPH>(m), &inverse);
                if (there) store_codes(cache + to, 8, fp8_codes(v, inverse));
                if (c == 0 && there) (which == 1 ? p.cache.k_scale : p.cache.v_scale)[scale_at + i * p.cache.scale_head_step] = s;
            } else if (there) {
                if (p.cache.type == NQ_KV_F16)
                    put8<_Float16>(cache, to, v);
                else
                    put8<bf16_t>(cache, to, v);
            }
        }
    }
}

template <typename T, int LPH>
static nq_status launch_lanes(HeadParams &p, hipStream_t s)
{
    const int per = 64 / LPH, most = (int)(ceil_div(p.Hq, per) + ceil_div(p.Hk, per) + ceil_div(p.Hv, per));
    // few tokens: their heads are dealt to several waves, which make the angles each (1024 tokens in one, two, four, eight: 12.1, 10.1, 9.4, 12.3 us)
    p.split = (int)std::max<int64_t>(1, std::min<int64_t>(most, 4096 / std::max<int64_t>(p.T, 1)));
    const int mode = p.rotary == 0 ? 0 : p.pairs == NQ_PAIRS_NEIGHBOURS ? 1 : LPH <= 16 && p.rotary == LPH * 8 ? 4 : p.rotary % 16 == 0 ? 2 : 3;
    for (p.first = 0; p.first < p.T; p.first = p.last) {             // (a dispatch has fewer than 2^32 threads)
        p.last = std::min(p.T, p.first + (int64_t(1) << 24));
        const dim3 grid((unsigned)ceil_div((p.last - p.first) * p.split, 4));
        if (mode == 0)
            k_head_norm<T, LPH, 0><<<grid, 256, 0, s>>>(p);
        else if (mode == 1)
            k_head_norm<T, LPH, 1><<<grid, 256, 0, s>>>(p);
        else if (mode == 2)
            k_head_norm<T, LPH, 2><<<grid, 256, 0, s>>>(p);
        else if (mode == 4) {
            if constexpr (LPH <= 16) k_head_norm<T, LPH, 4><<<grid, 256, 0, s>>>(p);
        } else
            k_head_norm<T, LPH, 3><<<grid, 256, 0, s>>>(p);
        const nq_status st = launch_status();
        if (st != NQ_OK) return st;
    }
    return NQ_OK;
}

template <typename T>
static nq_status launch_heads(HeadParams &p, hipStream_t s)
{
    if (p.D <= 64) return launch_lanes<T, 8>(p, s);
    return p.D <= 128 ? launch_lanes<T, 16>(p, s) : launch_lanes<T, 32>(p, s);
}

struct ReadParams {
    CacheView cache;
    const int64_t *slot;
    void *k, *v;
    int64_t ldk, ldv, first;               // first: row of this launch's first
    uint32_t count;                        // pieces of eight elements of this launch
    Divider by_pieces, by_heads;           // pieces of a head; heads
    int32_t D;
};

// Eight elements of a cache as they lie in memory (zeros: of no row).
struct Kept8 {
    uint4 w;
    float scale;
};
__device__ __forceinline__ Kept8 fetch_kept(const uint8_t *base, int64_t at, int type, const float *scale)
{
    Kept8 r{};
    if (type == NQ_KV_E4M3) {
        __builtin_memcpy(&r.w, base + at, 8);
        r.scale = *scale;
    } else {
        __builtin_memcpy(&r.w, base + at * 2, 16);
    }
    return r;
}
__device__ __forceinline__ void floats_of(const Kept8 &r, int type, float (&v)[8])
{
    if (type == NQ_KV_E4M3) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int d = (int)(i ? r.w.y : r.w.x);
            const f8_f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(d, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(d, true);
            v[4 * i] = a.x * r.scale;
            v[4 * i + 1] = a.y * r.scale;
            v[4 * i + 2] = b.x * r.scale;
            v[4 * i + 3] = b.y * r.scale;
        }
    } else if (type == NQ_KV_F16) {
        raw_to_float(Raw8<_Float16>{r.w}, v);
    } else {
        raw_to_float(Raw8<bf16_t>{r.w}, v);
    }
}

// A thread takes eight elements of a row's key and then of its value (32768 rows of 8 x 128 e4m3 to bf16 46.5 us, 4.5 TB/s, two thirds of it
// written; with both asked for before either is written 47.0).
template <typename T>
__global__ void __launch_bounds__(256) k_cache_read(const ReadParams p)
{
    const uint32_t id = blockIdx.x * 256u + threadIdx.x;
    if (id >= p.count) return;
    const uint32_t at = divide(id, p.by_pieces);
    const int c = (int)(id - at * p.by_pieces.d) * 8;
    const uint32_t r = divide(at, p.by_heads), h = at - r * p.by_heads.d;
    const int64_t t = p.first + r, slot = p.slot[t];
    const bool there = slot >= 0 && slot < p.cache.slots;
    const Place l = place_of(p.cache, there ? slot : 0);
    const int64_t from = l.page * p.cache.page_step + l.token * p.cache.token_step + h * p.cache.head_step + c;
    const int64_t scale = l.page * p.cache.scale_page_step + l.token * p.cache.scale_token_step + h * p.cache.scale_head_step;
    float x[8];
    if (p.k) {
        const Kept8 k = there ? fetch_kept(p.cache.k, from, p.cache.type, p.cache.k_scale + scale) : Kept8{};
        floats_of(k, p.cache.type, x);
        put8<T>(p.k, t * p.ldk + (int64_t)h * p.D + c, x);
    }
    if (p.v) {
        const Kept8 v = there ? fetch_kept(p.cache.v, from, p.cache.type, p.cache.v_scale + scale) : Kept8{};
        floats_of(v, p.cache.type, x);
        put8<T>(p.v, t * p.ldv + (int64_t)h * p.D + c, x);
    }
}

static nq_status check_head_norm(const nq_norm &n)
{
    if (n.kind < NQ_NORM_NONE || n.kind > NQ_NORM_LAYER) return NQ_ERR_INVALID_ARG;
    return aligned_to(n.d_weight, 4) && aligned_to(n.d_bias, 4) ? NQ_OK : NQ_ERR_ALIGN;
}

}  // namespace nq

using namespace nq;

extern "C" nq_status nq_head_norm(const nq_head_job *job, int64_t T, void *stream)
{
    if (!job || T < 0) return NQ_ERR_INVALID_ARG;
    const nq_head_job &j = *job;
    if (!is_dtype(j.dtype) || (j.pairs != NQ_PAIRS_HALVES && j.pairs != NQ_PAIRS_NEIGHBOURS)) return NQ_ERR_INVALID_ARG;
    nq_status st;
    if ((st = check_heads(j.q_heads, j.kv_heads, j.head_dim)) != NQ_OK) return st;
    if ((st = check_head_norm(j.q_norm)) != NQ_OK || (st = check_head_norm(j.k_norm)) != NQ_OK) return st;
    if (j.rotary < 0 || j.rotary % 2) return NQ_ERR_INVALID_ARG;
    if (j.rotary > j.head_dim || T > ATT_MAX_ROWS) return NQ_ERR_SHAPE;
    if (j.cache) {
        if ((st = check_cache(j.cache)) != NQ_OK) return st;
        if (j.cache->heads != j.kv_heads || j.cache->head_dim != j.head_dim) return NQ_ERR_SHAPE;
    }
    if (T == 0) return NQ_OK;
    const int64_t wq = (int64_t)j.q_heads * j.head_dim, wk = (int64_t)j.kv_heads * j.head_dim;
    if (j.d_q && (st = check_matrix(j.d_q, j.dtype, wq, j.ldq)) != NQ_OK) return st;
    if (j.d_q && (st = check_matrix(j.d_q_out, j.dtype, wq, j.ldq_out)) != NQ_OK) return st;
    if (j.d_k && (st = check_matrix(j.d_k, j.dtype, wk, j.ldk)) != NQ_OK) return st;
    if (j.d_k && j.d_k_out && (st = check_matrix(j.d_k_out, j.dtype, wk, j.ldk_out)) != NQ_OK) return st;
    if (j.d_v && (st = check_matrix(j.d_v, j.dtype, wk, j.ldv)) != NQ_OK) return st;
    if (j.cache && !j.d_slot) return NQ_ERR_INVALID_ARG;
    if (j.cache && !aligned_to(j.d_slot, 8)) return NQ_ERR_ALIGN;
    if (j.rotary && (!j.d_freq || !j.d_position)) return NQ_ERR_INVALID_ARG;
    if (j.rotary && (!aligned_to(j.d_freq, 4) || !aligned_to(j.d_position, 4))) return NQ_ERR_ALIGN;

    HeadParams p;
    p.q = j.d_q;
    p.k = j.d_k;
    p.v = j.d_v;
    p.q_out = j.d_q_out;
    p.k_out = j.d_k_out;
    p.ldq = j.ldq;
    p.ldk = j.ldk;
    p.ldv = j.ldv;
    p.ldq_out = j.ldq_out;
    p.ldk_out = j.ldk_out;
    // (the bias belongs to the layer norm alone)
    auto vector_of = [](const nq_norm &n, const float *v, bool bias) { return n.kind == NQ_NORM_NONE || (bias && n.kind == NQ_NORM_RMS) ? nullptr : v; };
    p.q_w = vector_of(j.q_norm, j.q_norm.d_weight, false);
    p.q_b = vector_of(j.q_norm, j.q_norm.d_bias, true);
    p.k_w = vector_of(j.k_norm, j.k_norm.d_weight, false);
    p.k_b = vector_of(j.k_norm, j.k_norm.d_bias, true);
    p.freq = j.d_freq;
    p.position = j.d_position;
    p.slot = j.d_slot;
    p.cached = j.cache && j.cache->pages > 0;
    p.cache = j.cache ? view_of(*j.cache) : CacheView{};
    p.T = T;
    p.q_eps = j.q_norm.eps;
    p.k_eps = j.k_norm.eps;
    p.inv_D = 1.0f / (float)j.head_dim;
    p.Hq = j.d_q ? j.q_heads : 0;
    p.Hk = j.d_k && (p.cached || j.d_k_out) ? j.kv_heads : 0;
    p.Hv = j.d_v && p.cached ? j.kv_heads : 0;
    p.q_kind = j.q_norm.kind;
    p.k_kind = j.k_norm.kind;
    p.D = j.head_dim;
    p.rotary = j.rotary;
    p.pairs = j.pairs;
    if (p.Hq + p.Hk + p.Hv == 0) return NQ_OK;
    hipStream_t s = (hipStream_t)stream;
    if (j.dtype == NQ_DT_F32) return launch_heads<float>(p, s);
    return j.dtype == NQ_DT_F16 ? launch_heads<_Float16>(p, s) : launch_heads<bf16_t>(p, s);
}

extern "C" nq_status nq_cache_read(const nq_kv_cache *cache, const int64_t *d_slot, int64_t T, void *d_k, int64_t ldk, void *d_v,
                                   int64_t ldv, int dtype, void *stream)
{
    if (!is_dtype(dtype) || T < 0) return NQ_ERR_INVALID_ARG;
    nq_status st = check_cache(cache);
    if (st != NQ_OK) return st;
    if (T > ATT_MAX_ROWS) return NQ_ERR_SHAPE;
    if (T == 0 || (!d_k && !d_v)) return NQ_OK;
    if (!d_slot) return NQ_ERR_INVALID_ARG;
    if (!aligned_to(d_slot, 8)) return NQ_ERR_ALIGN;
    const int64_t width = (int64_t)cache->heads * cache->head_dim;
    if (d_k && (st = check_matrix(d_k, dtype, width, ldk)) != NQ_OK) return st;
    if (d_v && (st = check_matrix(d_v, dtype, width, ldv)) != NQ_OK) return st;
    ReadParams p;
    p.cache = view_of(*cache);
    p.slot = d_slot;
    p.k = d_k;
    p.v = d_v;
    p.ldk = ldk;
    p.ldv = ldv;
    p.by_heads = make_divider((uint32_t)cache->heads);
    p.D = cache->head_dim;
    p.by_pieces = make_divider((uint32_t)cache->head_dim / 8);
    const int64_t pieces = width / 8, step = std::max<int64_t>(1, (int64_t(1) << 30) / pieces);      // (a dispatch has fewer than 2^32 threads)
    for (p.first = 0; p.first < T; p.first += step) {
        p.count = (uint32_t)(std::min(step, T - p.first) * pieces);
        const dim3 grid((unsigned)ceil_div(p.count, 256));
        if (dtype == NQ_DT_F32)
            k_cache_read<float><<<grid, 256, 0, (hipStream_t)stream>>>(p);
        else if (dtype == NQ_DT_F16)
            k_cache_read<_Float16><<<grid, 256, 0, (hipStream_t)stream>>>(p);
        else
            k_cache_read<bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(p);
        if ((st = launch_status()) != NQ_OK) return st;
    }
    return NQ_OK;
}
