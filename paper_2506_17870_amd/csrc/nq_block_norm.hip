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

// Sum over the workgroup, the same in every thread and every run: within the waves first, then the waves' sums in order.
template <int TH>
__device__ __forceinline__ float block_sum(float v, float *part)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    if constexpr (TH > 64) {
        __syncthreads();                               // (the last sum's readers are done)
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < TH / 64; ++i) v += part[i];
    }
    return v;
}

// v -> norm(v).  The variance is that of the differences from the mean (two sums over registers), not a difference of two
// large sums.
template <int TH, int NC>
__device__ __forceinline__ void norm_row(int kind, float eps, const float *__restrict__ w, const float *__restrict__ b, const int (&n)[NC],
                                         int D, bool vec, float (&v)[NC][8], float *part)
{
    if (kind == NQ_NORM_NONE) return;
    const float count = (float)D;
    if (kind == NQ_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[k][i];
        const float mean = block_sum<TH>(s, part) / count;
#pragma unroll
        for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = i < n[k] ? v[k][i] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(v[k][i], v[k][i], s);
    const float r = 1.0f / sqrtf(block_sum<TH>(s, part) / count + eps);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        const int c = (int)(threadIdx.x + k * TH) * 8;
        float wv[8], bv[8];
        if (w) raw_to_float(vec ? load8<true>(w + c, n[k]) : load8<false>(w + c, n[k]), wv);
        if (b) raw_to_float(vec ? load8<true>(b + c, n[k]) : load8<false>(b + c, n[k]), bv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[k][i] *= r;
            if (w) v[k][i] *= wv[i];
            if (b) v[k][i] += bv[i];
        }
    }
}

// TH threads to a row, NC times eight columns each.  VEC: every row of every operand starts on 16 bytes (codes: 8).
template <typename T, typename H, bool VEC, int TH, int NC>
__global__ void __launch_bounds__(TH) k_block_norm(const NormParams p)
{
    __shared__ float part[TH / 64];
    int n[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) n[k] = min(8, max(0, p.D - (int)(threadIdx.x + k * TH) * 8));
    const int c0 = threadIdx.x * 8;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        Raw8<H> hr[NC];
        Raw8<T> yr[NC], gr[NC];
        const T *gate = static_cast<const T *>(p.gate) + row / p.gate_rows * p.ldgate;
        auto load_h = [&](int k) {
            const int c = c0 + k * TH * 8;
            hr[k] = load8<VEC>(static_cast<const H *>(p.h) + row * p.ldh + c, n[k]);
            if (p.gate) gr[k] = load8<VEC>(gate + c, n[k]);
        };
        if (p.y) {
#pragma unroll
            for (int k = 0; k < NC; ++k) yr[k] = load8<VEC>(static_cast<const T *>(p.y) + row * p.ldy + c0 + k * TH * 8, n[k]);
        }
        // all requests of a row at once, where there are registers for it
        if constexpr (NC <= 2) {
#pragma unroll
            for (int k = 0; k < NC; ++k) load_h(k);
        }
        float v[NC][8];
        if (p.y) {
#pragma unroll
            for (int k = 0; k < NC; ++k) raw_to_float(yr[k], v[k]);
            norm_row<TH, NC>(p.post, p.post_eps, p.post_w, p.post_b, n, p.D, VEC, v, part);
        }
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            float h[8], g[8];
            if constexpr (NC > 2) load_h(k);
            raw_to_float(hr[k], h);
            if (p.gate) raw_to_float(gr[k], g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float d = 0.0f;
                if (p.y) d = p.branch_scale * (p.gate ? g[i] * v[k][i] : v[k][i]);
                v[k][i] = i < n[k] ? p.residual_scale * h[i] + d : 0.0f;
            }
            if (p.h_out) store8<VEC>(static_cast<H *>(p.h_out) + row * p.ldh_out + c0 + k * TH * 8, n[k], v[k]);
        }
        if (!p.x && !p.q) continue;
        norm_row<TH, NC>(p.pre, p.pre_eps, p.pre_w, p.pre_b, n, p.D, VEC, v, part);
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            const int c = c0 + k * TH * 8;
            if (p.x) store8<VEC>(static_cast<T *>(p.x) + row * p.ldx + c, n[k], v[k]);
            if (p.q) {
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) a = max(a, i < n[k] ? abs_bits(v[k][i]) : 0u);
                float inverse;
                const float s = fp8_scale(max16(a), &inverse);
                store_codes<VEC>(p.q + row * p.ldq + c, n[k], fp8_codes(v[k], inverse));
                if ((threadIdx.x & 15) == 0 && n[k] > 0) p.scale[row * p.srow + (c >> 7) * p.scol] = s;
            }
        }
    }
}

// Rows too long for the registers (D > 16384): the fp32 row lies in LDS, where a thread reads back only what it wrote itself.
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

template <bool VEC>
__device__ __forceinline__ void norm_long_row(const NormParams &p, f8_f4 *row, int kind, float eps, const float *__restrict__ w,
                                              const float *__restrict__ b, float *part)
{
    if (kind == NQ_NORM_NONE) return;
    const float count = (float)p.D;
    float s = 0.0f, mean = 0.0f;
    if (kind == NQ_NORM_LAYER) {
        long_row(p, row, [&](int, int, float (&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        });
        mean = block_sum<LONG_TH>(s, part) / count;
        s = 0.0f;
    }
    long_row(p, row, [&](int, int n, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = i < n ? v[i] - mean : 0.0f;
            s = fmaf(v[i], v[i], s);
        }
    });
    const float r = 1.0f / sqrtf(block_sum<LONG_TH>(s, part) / count + eps);
    long_row(p, row, [&](int c, int n, float (&v)[8]) {
        float wv[8], bv[8];
        if (w) raw_to_float(load8<VEC>(w + c, n), wv);
        if (b) raw_to_float(load8<VEC>(b + c, n), bv);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] *= r;
            if (w) v[i] *= wv[i];
            if (b) v[i] += bv[i];
        }
    });
}

template <typename T, typename H, bool VEC>
__global__ void __launch_bounds__(LONG_TH) k_block_norm_long(const NormParams p)
{
    extern __shared__ __attribute__((aligned(16))) f8_f4 lds[];
    __shared__ float part[LONG_TH / 64];
    for (int64_t r = blockIdx.x; r < p.M; r += gridDim.x) {
        const T *gate = static_cast<const T *>(p.gate) + r / p.gate_rows * p.ldgate;
        if (p.y) {
            long_row(p, lds, [&](int c, int n, float (&v)[8]) { raw_to_float(load8<VEC>(static_cast<const T *>(p.y) + r * p.ldy + c, n), v); });
            norm_long_row<VEC>(p, lds, p.post, p.post_eps, p.post_w, p.post_b, part);
        }
        long_row(p, lds, [&](int c, int n, float (&v)[8]) {
            float h[8], g[8];
            raw_to_float(load8<VEC>(static_cast<const H *>(p.h) + r * p.ldh + c, n), h);
            if (p.gate) raw_to_float(load8<VEC>(gate + c, n), g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float d = 0.0f;
                if (p.y) d = p.branch_scale * (p.gate ? g[i] * v[i] : v[i]);
                v[i] = i < n ? p.residual_scale * h[i] + d : 0.0f;
            }
            if (p.h_out) store8<VEC>(static_cast<H *>(p.h_out) + r * p.ldh_out + c, n, v);
        });
        if (!p.x && !p.q) continue;
        norm_long_row<VEC>(p, lds, p.pre, p.pre_eps, p.pre_w, p.pre_b, part);
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
            if (p.x) store8<VEC>(static_cast<T *>(p.x) + r * p.ldx + c, n, v);
            if (p.q) {
                float inverse;
                const float s = fp8_scale(max16(a), &inverse);
                store_codes<VEC>(p.q + r * p.ldq + c, n, fp8_codes(v, inverse));
                if ((threadIdx.x & 15) == 0) p.scale[r * p.srow + (c >> 7) * p.scol] = s;
            }
        }
    }
}

template <typename T, typename H, bool VEC, int TH, int NC>
static void launch_norm(const NormParams &p, hipStream_t s)
{
    k_block_norm<T, H, VEC, TH, NC><<<(unsigned)std::min<int64_t>(p.M, 1 << 20), TH, 0, s>>>(p);
}

template <typename T, typename H, bool VEC>
static void launch_norm_long(const NormParams &p, hipStream_t s)
{
    const int lds = (p.D + 7) / 8 * 32;
    auto k = k_block_norm_long<T, H, VEC>;
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    k<<<(unsigned)std::min<int64_t>(p.M, 1 << 20), LONG_TH, lds, s>>>(p);
}

template <typename T, typename H, bool VEC>
static void norm_by_size(const NormParams &p, hipStream_t s)
{
    const int chunks = (p.D + 7) / 8;
    if (chunks <= 64)
        launch_norm<T, H, VEC, 64, 1>(p, s);
    else if (chunks <= 128)
        launch_norm<T, H, VEC, 128, 1>(p, s);
    else if (chunks <= 256)
        launch_norm<T, H, VEC, 256, 1>(p, s);
    else if (chunks <= 512)
        launch_norm<T, H, VEC, 256, 2>(p, s);
    else if (chunks <= 1024)
        launch_norm<T, H, VEC, 512, 2>(p, s);
    else if (chunks <= 2048)
        launch_norm<T, H, VEC, 512, 4>(p, s);
    else
        launch_norm_long<T, H, VEC>(p, s);
}

template <typename T, typename H>
static void norm_by_alignment(const NormParams &p, bool vec, hipStream_t s)
{
    if (vec)
        norm_by_size<T, H, true>(p, s);
    else
        norm_by_size<T, H, false>(p, s);
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
    const bool vec = rows_on_16(p.h, j.h_dtype, p.ldh) && rows_on_16(p.y, j.dtype, p.ldy) && rows_on_16(p.gate, j.dtype, p.ldgate) &&
                     rows_on_16(p.h_out, j.h_dtype, p.ldh_out) && rows_on_16(p.x, j.dtype, p.ldx) && aligned16(p.post_w) &&
                     aligned16(p.post_b) && aligned16(p.pre_w) && aligned16(p.pre_b) && aligned_to(p.q, 8) && p.ldq % 8 == 0;
    hipStream_t s = (hipStream_t)stream;
    if (j.dtype == NQ_DT_F32)
        norm_by_alignment<float, float>(p, vec, s);
    else if (j.dtype == NQ_DT_F16 && j.h_dtype == NQ_DT_F16)
        norm_by_alignment<_Float16, _Float16>(p, vec, s);
    else if (j.dtype == NQ_DT_F16)
        norm_by_alignment<_Float16, float>(p, vec, s);
    else if (j.h_dtype == NQ_DT_BF16)
        norm_by_alignment<bf16_t, bf16_t>(p, vec, s);
    else
        norm_by_alignment<bf16_t, float>(p, vec, s);
    return launch_status();
}
