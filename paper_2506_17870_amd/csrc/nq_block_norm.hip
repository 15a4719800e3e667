// nq_block_norm: the norm after a block, its gate, the residual sum and the norm before the next block in one pass over the
// rows.  Bound by the bytes (h, y, the gate in; h' and x out, each once); a row stays in the registers of one workgroup from
// its first statistic to its last store, so neither the branch nor the new stream is read back.
#include "nq_fp8.h"

namespace nq {

struct NormParams {
    const void *h, *y, *gate;
    void *h_out, *x;
    const float *post_w, *post_b, *pre_w, *pre_b;
    uint8_t *q;
    float *scale;
    int64_t ldh, ldy, ldgate, ldh_out, ldx, ldq, srow, scol, M, gate_rows;
    float residual_scale, branch_scale, post_eps, pre_eps;
    int post, pre, D;
};

// Sum over the workgroup, the same in every thread and every run: within the waves first, then the waves' sums in order.  The
// sums of a row alternate between two sets of memory, so that one barrier each is enough: a wave that writes a set again has
// passed the barrier of the sum between, and with it every wave that still had to read it.
template <int TH>
struct BlockSum {
    float (*part)[TH / 64];
    int set;
    __device__ __forceinline__ float operator()(float v)
    {
        v = sum64(v);
        if constexpr (TH > 64) {
            if ((threadIdx.x & 63) == 0) part[set][threadIdx.x >> 6] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int i = 0; i < TH / 64; ++i) v += part[set][i];
            set ^= 1;
        }
        return v;
    }
};

// 1 / sqrt(x), the hardware's (good to a unit) also where x is too small for it.
__device__ __forceinline__ float inverse_root(float x)
{
    const bool small = x < 0x1p-100f;
    const float r = __builtin_amdgcn_rsqf(small ? x * 0x1p80f : x);
    return small ? r * 0x1p40f : r;
}

// The weights and biases of a norm for a thread's columns, in registers for all its rows.
template <bool FULL>
struct NormVectors {
    const float *w, *b;
    float wv[8], bv[8];
    __device__ __forceinline__ void init(const float *w_, const float *b_, int D, float b_scale)
    {
        w = w_;
        b = b_;
        if (w) raw_to_float(load8<FULL>(w, threadIdx.x * 8, D), wv);
        if (b) {
            raw_to_float(load8<FULL>(b, threadIdx.x * 8, D), bv);
#pragma unroll
            for (int i = 0; i < 8; ++i) bv[i] *= b_scale;
        }
    }
    __device__ __forceinline__ void apply(float r, float (&v)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= r;
        if (w) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= wv[i];
        }
        if (b) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += bv[i];
        }
    }
};

// v -> norm(v) * scale (the biases have it already).  The variance is that of the differences from the mean (two sums over registers),
// not a difference of two large sums.
template <int TH, bool FULL>
__device__ __forceinline__ void norm_row(int kind, float eps, float scale, NormVectors<FULL> &vec, int n, float per_column, float (&v)[8],
                                         BlockSum<TH> &sum)
{
    float r = 1.0f;
    if (kind != NQ_NORM_NONE) {
        if (kind == NQ_NORM_LAYER) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
            const float mean = sum(s) * per_column;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = FULL || i < n ? v[i] - mean : 0.0f;
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
        r = inverse_root(fmaf(sum(s), per_column, eps));
    }
    vec.apply(r * scale, v);
}

// A row to a workgroup of TH threads, eight columns to a thread; FULL: D is exactly 8 * TH.  A workgroup takes rows blockIdx.x,
// + gridDim.x, ...: the norms' vectors stay in its registers, and the next row is on its way while one is worked on.  (Columns past D
// read as zeros and stay zeros, so only the differences from a mean are masked.)  With eight columns to a thread the vector unit and
// the memory take about as long: every division, every mask and every conversion twice over that was taken out of the loop
// showed (16384 x 4096 bf16 to codes 123 -> 92 us, 5.1 TB/s, what a copy reaches).
template <typename T, typename H, int TH, bool FULL>
__global__ void __launch_bounds__(TH) k_block_norm(const NormParams p)
{
    __shared__ float part[2][TH / 64];
    BlockSum<TH> sum{part, 0};
    const int c = threadIdx.x * 8, n = FULL ? 8 : p.D - c;
    const float per_column = 1.0f / (float)p.D;

    struct Row {
        Raw8<T> y, g;
        Raw8<H> h;
    };
    auto load = [&](Row &r, int64_t row) {
        if (p.y) r.y = load8<FULL>(static_cast<const T *>(p.y) + row * p.ldy, c, p.D);
        r.h = load8<FULL>(static_cast<const H *>(p.h) + row * p.ldh, c, p.D);
        if (p.gate) r.g = load8<FULL>(static_cast<const T *>(p.gate) + row / p.gate_rows * p.ldgate, c, p.D);
    };
    Row now;
    load(now, blockIdx.x);
    NormVectors<FULL> post, pre;
    post.init(p.post_w, p.post_b, p.D, p.branch_scale);
    pre.init(p.pre_w, p.pre_b, p.D, 1.0f);

    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        Row next;
        if (row + gridDim.x < p.M) load(next, row + gridDim.x);
        float v[8] = {}, h[8];
        if (p.y) {
            raw_to_float(now.y, v);
            norm_row<TH, FULL>(p.post, p.post_eps, p.branch_scale, post, n, per_column, v, sum);
            if (p.gate) {
                float g[8];
                raw_to_float(now.g, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= g[i];
            }
        }
        raw_to_float(now.h, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(p.residual_scale, h[i], v[i]);
        if (p.h_out) store8(static_cast<H *>(p.h_out) + row * p.ldh_out + c, n, v);
        if (p.x || p.q) {
            norm_row<TH, FULL>(p.pre, p.pre_eps, 1.0f, pre, n, per_column, v, sum);
            if (p.x) store8(static_cast<T *>(p.x) + row * p.ldx + c, n, v);
            if (p.q) {
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) a = max(a, abs_bits(v[i]));
                float inverse;
                const float s = fp8_scale(max16(a), &inverse);
                store_codes(p.q + row * p.ldq + c, n, fp8_codes(v, inverse));
                if ((threadIdx.x & 15) == 0 && n > 0) p.scale[row * p.srow + (c >> 7) * p.scol] = s;
            }
        }
        now = next;
    }
}

// Rows too long for the registers (D > 8192): the fp32 row lies in LDS, where a thread reads back only what it wrote itself.
constexpr int LONG_TH = 512;

template <typename F>
__device__ __forceinline__ void long_row(const NormParams &p, f8_f4 *row, const F &f)
{
    for (int c = threadIdx.x * 8; c < p.D; c += LONG_TH * 8) {
        const int n = min(8, p.D - c);
        f8_f4 *at = row + (c >> 2);
        float v[8] = {at[0][0], at[0][1], at[0][2], at[0][3], at[1][0], at[1][1], at[1][2], at[1][3]};
        f(c, n, v);
        at[0] = f8_f4{v[0], v[1], v[2], v[3]};
        at[1] = f8_f4{v[4], v[5], v[6], v[7]};
    }
}

__device__ __forceinline__ void norm_long_row(const NormParams &p, f8_f4 *row, int kind, float eps, const float *__restrict__ w,
                                              const float *__restrict__ b, BlockSum<LONG_TH> &sum)
{
    if (kind == NQ_NORM_NONE) return;
    const float count = (float)p.D;
    float s = 0.0f, mean = 0.0f;
    if (kind == NQ_NORM_LAYER) {
        long_row(p, row, [&](int, int, float (&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        });
        mean = sum(s) / count;
        s = 0.0f;
    }
    long_row(p, row, [&](int, int n, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = i < n ? v[i] - mean : 0.0f;
            s = fmaf(v[i], v[i], s);
        }
    });
    const float r = inverse_root(sum(s) / count + eps);
    long_row(p, row, [&](int c, int n, float (&v)[8]) {
        float wv[8], bv[8];
        if (w) raw_to_float(load8<false>(w, c, p.D), wv);
        if (b) raw_to_float(load8<false>(b, c, p.D), bv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] *= r;
            if (w) v[i] *= wv[i];
            if (b) v[i] += bv[i];
        }
    });
}

template <typename T, typename H>
__global__ void __launch_bounds__(LONG_TH) k_block_norm_long(const NormParams p)
{
    extern __shared__ __attribute__((aligned(16))) f8_f4 lds[];
    __shared__ float part[2][LONG_TH / 64];
    BlockSum<LONG_TH> sum{part, 0};
    for (int64_t r = blockIdx.x; r < p.M; r += gridDim.x) {
        const T *gate = static_cast<const T *>(p.gate) + r / p.gate_rows * p.ldgate;
        if (p.y) {
            long_row(p, lds, [&](int c, int, float (&v)[8]) { raw_to_float(load8<false>(static_cast<const T *>(p.y) + r * p.ldy, c, p.D), v); });
            norm_long_row(p, lds, p.post, p.post_eps, p.post_w, p.post_b, sum);
        }
        long_row(p, lds, [&](int c, int n, float (&v)[8]) {
            float h[8], g[8];
            raw_to_float(load8<false>(static_cast<const H *>(p.h) + r * p.ldh, c, p.D), h);
            if (p.gate) raw_to_float(load8<false>(gate, c, p.D), g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float d = 0.0f;
                if (p.y) d = p.branch_scale * (p.gate ? g[i] * v[i] : v[i]);
                v[i] = i < n ? p.residual_scale * h[i] + d : 0.0f;
            }
            if (p.h_out) store8(static_cast<H *>(p.h_out) + r * p.ldh_out + c, n, v);
        });
        if (!p.x && !p.q) continue;
        norm_long_row(p, lds, p.pre, p.pre_eps, p.pre_w, p.pre_b, sum);
        // (whole blocks of 128 columns, so that all sixteen threads of one take part in its maximum)
        for (int c = threadIdx.x * 8; c < (p.D + 127) / 128 * 128; c += LONG_TH * 8) {
            const int n = min(8, max(0, p.D - c));
            float v[8];
            uint32_t a = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = i < n ? lds[(c + i) >> 2][i & 3] : 0.0f;
                a = max(a, abs_bits(v[i]));
            }
            if (p.x) store8(static_cast<T *>(p.x) + r * p.ldx + c, n, v);
            if (p.q) {
                float inverse;
                const float s = fp8_scale(max16(a), &inverse);
                store_codes(p.q + r * p.ldq + c, n, fp8_codes(v, inverse));
                if ((threadIdx.x & 15) == 0) p.scale[r * p.srow + (c >> 7) * p.scol] = s;
            }
        }
    }
}

template <typename T, typename H, int TH>
static void launch_norm(const NormParams &p, hipStream_t s)
{
    // up to sixteen waves to a compute unit (8: 126 us, 24: 103 us on the rows above)
    const dim3 grid((unsigned)std::min<int64_t>(p.M, 256 * (1024 / TH)));
    if (p.D == TH * 8)
        k_block_norm<T, H, TH, true><<<grid, TH, 0, s>>>(p);
    else
        k_block_norm<T, H, TH, false><<<grid, TH, 0, s>>>(p);
}

template <typename T, typename H>
static void norm_by_size(const NormParams &p, hipStream_t s)
{
    const int chunks = (p.D + 7) / 8;
    if (chunks <= 64) return launch_norm<T, H, 64>(p, s);
    if (chunks <= 128) return launch_norm<T, H, 128>(p, s);
    if (chunks <= 256) return launch_norm<T, H, 256>(p, s);
    if (chunks <= 384) return launch_norm<T, H, 384>(p, s);
    if (chunks <= 512) return launch_norm<T, H, 512>(p, s);
    if (chunks <= 768) return launch_norm<T, H, 768>(p, s);
    if (chunks <= 1024) return launch_norm<T, H, 1024>(p, s);
    const int lds = chunks * 32;
    auto k = k_block_norm_long<T, H>;
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    k<<<(unsigned)std::min<int64_t>(p.M, 1 << 20), LONG_TH, lds, s>>>(p);
}

static nq_status check_norm(const nq_norm &n)
{
    if (n.kind < NQ_NORM_NONE || n.kind > NQ_NORM_LAYER) return NQ_ERR_INVALID_ARG;
    return aligned_to(n.d_weight, 4) && aligned_to(n.d_bias, 4) ? NQ_OK : NQ_ERR_ALIGN;
}

}  // namespace nq

using namespace nq;

extern "C" nq_status nq_block_norm(const nq_norm_job *job, int64_t M, int64_t D, void *stream)
{
    if (!job || M < 0 || D < 1) return NQ_ERR_INVALID_ARG;
    const nq_norm_job &j = *job;
    if (!is_dtype(j.dtype) || !is_dtype(j.h_dtype)) return NQ_ERR_INVALID_ARG;
    if (j.h_dtype != j.dtype && j.h_dtype != NQ_DT_F32) return NQ_ERR_UNSUPPORTED;
    if (D > NQ_NORM_MAX_D || M > FP8_MAX_ROWS) return NQ_ERR_SHAPE;
    nq_status st;
    if ((st = check_norm(j.post)) != NQ_OK || (st = check_norm(j.pre)) != NQ_OK) return st;
    if (j.q) {
        if ((st = check_fp8(j.q)) != NQ_OK) return st;
        if (j.q->block_rows != 1) return NQ_ERR_UNSUPPORTED;
        if (j.q->rows != M || j.q->cols != D) return NQ_ERR_SHAPE;
    }
    if (M == 0) return NQ_OK;
    if ((st = check_matrix(j.d_h, j.h_dtype, D, j.ldh)) != NQ_OK) return st;
    if (j.d_y && (st = check_matrix(j.d_y, j.dtype, D, j.ldy)) != NQ_OK) return st;
    if (j.d_gate) {
        if (j.gate_rows < 1) return NQ_ERR_INVALID_ARG;
        if ((st = check_matrix(j.d_gate, j.dtype, D, j.ldgate)) != NQ_OK) return st;
    }
    if (j.d_h_out && (st = check_matrix(j.d_h_out, j.h_dtype, D, j.ldh_out)) != NQ_OK) return st;
    if (j.d_x && (st = check_matrix(j.d_x, j.dtype, D, j.ldx)) != NQ_OK) return st;
    if (!j.d_h_out && !j.d_x && !j.q) return NQ_OK;

    NormParams p;
    p.h = j.d_h;
    p.y = j.d_y;
    p.gate = j.d_y ? j.d_gate : nullptr;
    p.h_out = j.d_h_out;
    p.x = j.d_x;
    auto vector_of = [](const nq_norm &n, const float *v) { return n.kind == NQ_NORM_NONE ? nullptr : v; };
    p.post_w = vector_of(j.post, j.post.d_weight);
    p.post_b = vector_of(j.post, j.post.d_bias);
    p.pre_w = vector_of(j.pre, j.pre.d_weight);
    p.pre_b = vector_of(j.pre, j.pre.d_bias);
    // (the bias belongs to the layer norm alone)
    if (j.post.kind == NQ_NORM_RMS) p.post_b = nullptr;
    if (j.pre.kind == NQ_NORM_RMS) p.pre_b = nullptr;
    p.q = j.q ? j.q->d_q : nullptr;
    p.scale = j.q ? j.q->d_scale : nullptr;
    p.ldq = j.q ? j.q->ld : 0;
    p.srow = j.q ? j.q->scale_row_step : 0;
    p.scol = j.q ? j.q->scale_col_step : 0;
    p.ldh = j.ldh;
    p.ldy = j.ldy;
    p.ldgate = j.ldgate;
    p.ldh_out = j.ldh_out;
    p.ldx = j.ldx;
    p.M = M;
    p.gate_rows = p.gate ? j.gate_rows : 1;
    p.residual_scale = j.residual_scale;
    p.branch_scale = j.branch_scale;
    p.post_eps = j.post.eps;
    p.pre_eps = j.pre.eps;
    p.post = j.d_y ? j.post.kind : NQ_NORM_NONE;
    p.pre = j.pre.kind;
    p.D = (int)D;
    hipStream_t s = (hipStream_t)stream;
    if (j.dtype == NQ_DT_F32)
        norm_by_size<float, float>(p, s);
    else if (j.dtype == NQ_DT_F16 && j.h_dtype == NQ_DT_F16)
        norm_by_size<_Float16, _Float16>(p, s);
    else if (j.dtype == NQ_DT_F16)
        norm_by_size<_Float16, float>(p, s);
    else if (j.h_dtype == NQ_DT_BF16)
        norm_by_size<bf16_t, bf16_t>(p, s);
    else
        norm_by_size<bf16_t, float>(p, s);
    return launch_status();
}
