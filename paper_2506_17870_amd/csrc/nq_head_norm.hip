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
    int64_t T;
    float q_eps, k_eps, inv_D;
    int32_t Hq, Hk, Hv;                    // (0 for what is not there)
    int32_t q_kind, k_kind, D, rotary, pairs, cached;
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

// A workgroup takes a token, LPH lanes of eight values a head.  The angles are made once for all heads of the token.
template <typename T, int LPH>
__global__ void __launch_bounds__(256) k_head_norm(const HeadParams p)
{
    __shared__ float2 turn[NQ_HEAD_MAX_DIM / 2];
    __shared__ float stage[256 * 8];
    const int groups = blockDim.x / LPH, c = (threadIdx.x % LPH) * 8, half = p.rotary >> 1;
    float *mine = stage + (threadIdx.x / LPH) * LPH * 8;          // this head's values (only its own lanes touch them)
    const bool in = c < p.D;
    const int heads = p.Hq + p.Hk + p.Hv;
    for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
        if (half) {
            __syncthreads();                                      // (the last token's readers)
            const int32_t position = p.position[t];
            for (int i = threadIdx.x; i < half; i += blockDim.x) turn[i] = turn_of(position, p.freq[i]);
            __syncthreads();
        }
        int64_t slot = p.cached ? p.slot[t] : -1, at = 0, scale_at = 0;
        if (slot >= p.cache.slots) slot = -1;
        if (slot >= 0) {
            const Place l = place_of(p.cache, slot);
            at = l.page * p.cache.page_step + l.token * p.cache.token_step;
            scale_at = l.page * p.cache.scale_page_step + l.token * p.cache.scale_token_step;
        }
        for (int h = blockIdx.y * groups + threadIdx.x / LPH; h < heads; h += gridDim.y * groups) {
            const int which = h < p.Hq ? 0 : h < p.Hq + p.Hk ? 1 : 2, i = which == 0 ? h : which == 1 ? h - p.Hq : h - p.Hq - p.Hk;
            const void *from = which == 0 ? p.q : which == 1 ? p.k : p.v;
            const int64_t ld = which == 0 ? p.ldq : which == 1 ? p.ldk : p.ldv;
            Raw8<T> raw{};
            if (in) __builtin_memcpy(&raw, static_cast<const T *>(from) + t * ld + (int64_t)i * p.D + c, sizeof raw);
            float v[8];
            raw_to_float(raw, v);
            if (which < 2) {
                const int kind = which ? p.k_kind : p.q_kind;
                const float *w = which ? p.k_w : p.q_w, *b = which ? p.k_b : p.q_b;
                if (kind != NQ_NORM_NONE) {
                    float sum = 0.0f;
                    if (kind == NQ_NORM_LAYER) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum += v[e];
                        const float mean = sum_lanes<LPH>(sum) * p.inv_D;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = in ? v[e] - mean : 0.0f;
                        sum = 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
                    const float r = 1.0f / sqrtf(sum_lanes<LPH>(sum) * p.inv_D + (which ? p.k_eps : p.q_eps));
                    float x[8];
                    if (w && in) {
                        __builtin_memcpy(x, w + c, sizeof x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = v[e] * r * x[e];
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= r;
                    }
                    if (b && in) {
                        __builtin_memcpy(x, b + c, sizeof x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += x[e];
                    }
                }
                if (half) {
                    if (p.pairs == NQ_PAIRS_NEIGHBOURS) {
#pragma unroll
                        for (int e = 0; e < 8; e += 2)
                            if (c + e < p.rotary) {
                                const float2 u = turn[(c + e) >> 1];
                                const float a = v[e], b2 = v[e + 1];
                                v[e] = fmaf(a, u.x, -(b2 * u.y));
                                v[e + 1] = fmaf(b2, u.x, a * u.y);
                            }
                    } else {
                        __builtin_memcpy(mine + c, v, sizeof v);
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        __builtin_amdgcn_wave_barrier();          // (LDS serves a wave's requests in order)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int d = c + e;
                            if (d < half) {
                                const float2 u = turn[d];
                                v[e] = fmaf(v[e], u.x, -(mine[d + half] * u.y));
                            } else if (d < p.rotary) {
                                const float2 u = turn[d - half];
                                v[e] = fmaf(v[e], u.x, mine[d - half] * u.y);
                            }
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                    }
                }
                if (which == 0) {
                    if (in) put8<T>(p.q_out, t * p.ldq_out + (int64_t)i * p.D + c, v);
                    continue;
                }
                if (p.k_out && in) put8<T>(p.k_out, t * p.ldk_out + (int64_t)i * p.D + c, v);
            }
            if (slot < 0) continue;
            uint8_t *cache = which == 1 ? p.cache.k : p.cache.v;
            const int64_t to = at + i * p.cache.head_step + c;
            if (p.cache.type == NQ_KV_E4M3) {
                uint32_t a = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) a = max(a, in ? abs_bits(v[e]) : 0u);
                float inverse;
                const float s = fp8_scale(max_lanes<LPH>(a), &inverse);
                if (in) store_codes(cache + to, 8, fp8_codes(v, inverse));
                if (c == 0) (which == 1 ? p.cache.k_scale : p.cache.v_scale)[scale_at + i * p.cache.scale_head_step] = s;
            } else if (in) {
                if (p.cache.type == NQ_KV_F16)
                    put8<_Float16>(cache, to, v);
                else
                    put8<bf16_t>(cache, to, v);
            }
        }
    }
}

template <typename T>
static nq_status launch_heads(const HeadParams &p, hipStream_t s)
{
    const int lph = p.D <= 64 ? 8 : p.D <= 128 ? 16 : 32, heads = p.Hq + p.Hk + p.Hv;
    const int threads = (int)std::min<int64_t>(256, round_up((int64_t)heads * lph, 64)), groups = threads / lph;
    // few tokens: their heads are dealt to several workgroups, which make the angles each
    const int split = p.T < 512 ? (int)ceil_div(heads, groups) : 1;
    const dim3 grid((unsigned)std::min<int64_t>(p.T, 1 << 22), split);
    if (lph == 8)
        k_head_norm<T, 8><<<grid, threads, 0, s>>>(p);
    else if (lph == 16)
        k_head_norm<T, 16><<<grid, threads, 0, s>>>(p);
    else
        k_head_norm<T, 32><<<grid, threads, 0, s>>>(p);
    return launch_status();
}

struct ReadParams {
    CacheView cache;
    const int64_t *slot;
    void *k, *v;
    int64_t ldk, ldv, first;               // first: row of this launch's first
    uint32_t count;                        // rows * heads of this launch
    Divider by_heads;
    int32_t D;
};

template <typename T>
__device__ __forceinline__ void read8(const uint8_t *base, int64_t at, int type, const float *scale, bool there, T *to)
{
    float v[8] = {};
    if (there) {
        if (type == NQ_KV_E4M3) {
            uint2 q;
            __builtin_memcpy(&q, base + at, 8);
            const float s = *scale;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int d = (int)(i ? q.y : q.x);
                const f8_f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(d, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(d, true);
                v[4 * i] = a.x * s;
                v[4 * i + 1] = a.y * s;
                v[4 * i + 2] = b.x * s;
                v[4 * i + 3] = b.y * s;
            }
        } else if (type == NQ_KV_F16) {
            Raw8<_Float16> r;
            __builtin_memcpy(&r, reinterpret_cast<const _Float16 *>(base) + at, 16);
            raw_to_float(r, v);
        } else {
            Raw8<bf16_t> r;
            __builtin_memcpy(&r, reinterpret_cast<const bf16_t *>(base) + at, 16);
            raw_to_float(r, v);
        }
    }
    store8(to, 8, v);
}

// LPH lanes of eight values take a head of a row, its key and its value.
template <typename T, int LPH>
__global__ void __launch_bounds__(256) k_cache_read(const ReadParams p)
{
    const uint32_t at = blockIdx.x * (256u / LPH) + threadIdx.x / LPH;
    const int c = (threadIdx.x % LPH) * 8;
    if (at >= p.count || c >= p.D) return;
    const uint32_t r = divide(at, p.by_heads), h = at - r * p.by_heads.d;
    const int64_t t = p.first + r, slot = p.slot[t];
    const bool there = slot >= 0 && slot < p.cache.slots;
    const Place l = place_of(p.cache, there ? slot : 0);
    const int64_t from = l.page * p.cache.page_step + l.token * p.cache.token_step + h * p.cache.head_step + c;
    const int64_t scale = l.page * p.cache.scale_page_step + l.token * p.cache.scale_token_step + h * p.cache.scale_head_step;
    if (p.k) read8(p.cache.k, from, p.cache.type, p.cache.k_scale + scale, there, static_cast<T *>(p.k) + t * p.ldk + (int64_t)h * p.D + c);
    if (p.v) read8(p.cache.v, from, p.cache.type, p.cache.v_scale + scale, there, static_cast<T *>(p.v) + t * p.ldv + (int64_t)h * p.D + c);
}

template <typename T>
static void launch_read(const ReadParams &p, hipStream_t s)
{
    if (p.D <= 64)
        k_cache_read<T, 8><<<(p.count + 31) / 32, 256, 0, s>>>(p);
    else if (p.D <= 128)
        k_cache_read<T, 16><<<(p.count + 15) / 16, 256, 0, s>>>(p);
    else
        k_cache_read<T, 32><<<(p.count + 7) / 8, 256, 0, s>>>(p);
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
    // (a dispatch has fewer than 2^32 threads, 32 at most to a head of a row)
    const int64_t step = (int64_t(1) << 26) / cache->heads;
    for (p.first = 0; p.first < T; p.first += step) {
        p.count = (uint32_t)(std::min(step, T - p.first) * cache->heads);
        if (dtype == NQ_DT_F32)
            launch_read<float>(p, (hipStream_t)stream);
        else if (dtype == NQ_DT_F16)
            launch_read<_Float16>(p, (hipStream_t)stream);
        else
            launch_read<bf16_t>(p, (hipStream_t)stream);
        if ((st = launch_status()) != NQ_OK) return st;
    }
    return NQ_OK;
}
