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

// Sum over the TH threads of a row, the same in every one and every run: within the waves first, then the waves' sums in order.  The
// sums of a row alternate between two sets of memory, so that one barrier each is enough: a wave that writes a set again has
// passed the barrier of the sum between, and with it every wave that still had to read it.
template <int TH>
struct BlockSum {
    float (*part)[TH < 64 ? 1 : TH / 64];
    int set;
    __device__ __forceinline__ float operator()(float v)
    {
        if constexpr (TH < 64) {
            v = sum16(v);
            return TH == 16 ? v : v + __shfl_xor(v, 16);
        }
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

// The weights and biases of a norm for a thread's columns: in registers for all its rows where it has eight columns, else read for
// every row (they stay in the caches).
template <int FIT, int CH>
struct NormVectors {
    const float *w, *b;
    int D;
    float b_scale, wv[8], bv[8];
    __device__ __forceinline__ void read(int c)
    {
        if (w) raw_to_float(load8<FIT>(w, c, D), wv);
        if (b) {
            raw_to_float(load8<FIT>(b, c, D), bv);
#pragma unroll
            for (int i = 0; i < 8; ++i) bv[i] *= b_scale;
        }
    }
    __device__ __forceinline__ void init(const float *w_, const float *b_, int c, int D_, float b_scale_)
    {
        w = w_;
        b = b_;
        D = D_;
        b_scale = b_scale_;
        if constexpr (CH == 1) read(c);
    }
    __device__ __forceinline__ void apply(float r, int c, float (&v)[8])
    {
        if constexpr (CH > 1) read(c);
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
template <int TH, int FIT, int CH>
__device__ __forceinline__ void norm_row(int kind, float eps, float scale, NormVectors<FIT, CH> &vec, int c, int D, float per_column,
                                         float (&v)[CH][8], BlockSum<TH> &sum)
{
    float r = 1.0f;
    if (kind != NQ_NORM_NONE) {
        if (kind == NQ_NORM_LAYER) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8 * CH; ++i) s += v[i / 8][i % 8];
            const float mean = sum(s) * per_column;
#pragma unroll
            for (int i = 0; i < 8 * CH; ++i) {
                float &x = v[i / 8][i % 8];
                x = FIT == FULL || c + i / 8 * TH * 8 + (FIT == WHOLE ? 0 : i % 8) < D ? x - mean : 0.0f;
            }
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8 * CH; ++i) s = fmaf(v[i / 8][i % 8], v[i / 8][i % 8], s);
        r = inverse_root(fmaf(sum(s), per_column, eps));
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        vec.apply(r * scale, c + k * TH * 8, v[k]);
        if (CH > 1) __builtin_amdgcn_sched_barrier(0);       // (one chunk's vectors at a time: registers)
    }
}

// A row to TH threads, CH times eight columns to a thread.  A workgroup takes rows blockIdx.x,
// + gridDim.x, ...: the norms' vectors stay in its registers, and the next row is on its way while one is worked on.  (Columns past D
// read as zeros and stay zeros, so only the differences from a mean are masked.)  With eight columns to a thread the vector unit and
// the memory take about as long: every division, every mask and every conversion twice over that was taken out of the loop
// showed (16384 x 4096 bf16 to codes 123 -> 86 us, 5.4 TB/s, what a copy reaches).  Rows of 256 columns at most share the waves of a
// workgroup of 256 threads (16054 x 128 f16 to codes 11.5 -> 5.1 us).  Rows that do not fit 1024 threads have sixteen columns to
// one; the next row is asked for when the stream's new row is formed, with 1024 threads at the end, when its registers are free
// (4096 x 16384 bf16 to codes 156 -> 98 us against the row in LDS).
constexpr int norm_rows(int th) { return th < 64 ? 256 / th : 1; }       // rows that a workgroup has at once

template <typename T, typename H, int TH, int CH, int FIT>
__global__ void __launch_bounds__(TH * norm_rows(TH)) k_block_norm(const NormParams p)
{
    constexpr int ROWS = norm_rows(TH);
    __shared__ float part[2][TH < 64 ? 1 : TH / 64];
    BlockSum<TH> sum{part, 0};
    const int c = (ROWS == 1 ? threadIdx.x : threadIdx.x % TH) * 8;
    const int64_t first = (int64_t)blockIdx.x * ROWS + (ROWS == 1 ? 0 : threadIdx.x / TH), step = (int64_t)gridDim.x * ROWS;
    if (ROWS > 1 && first >= p.M) return;
    const float per_column = 1.0f / (float)p.D;
    auto left = [&](int k) {
        const int n = p.D - (c + k * TH * 8);
        return FIT == CUT ? n : FIT == FULL || n > 0 ? 8 : 0;
    };

    struct Row {
        Raw8<T> y[CH], g[CH];
        Raw8<H> h[CH];
    };
    auto load = [&](Row &r, int64_t row) {
        const T *y = static_cast<const T *>(p.y) + row * p.ldy;
        const H *h = static_cast<const H *>(p.h) + row * p.ldh;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (p.y) r.y[k] = fetch8<FIT>(y, c + k * TH * 8, p.D);
            r.h[k] = fetch8<FIT>(h, c + k * TH * 8, p.D);
        }
        if (p.gate) {
            const T *gate = static_cast<const T *>(p.gate) + row / p.gate_rows * p.ldgate;
#pragma unroll
            for (int k = 0; k < CH; ++k) r.g[k] = fetch8<FIT>(gate, c + k * TH * 8, p.D);
        }
    };
    Row now;
    load(now, first);
    NormVectors<FIT, CH> post, pre;
    post.init(p.post_w, p.post_b, c, p.D, p.branch_scale);
    pre.init(p.pre_w, p.pre_b, c, p.D, 1.0f);

    for (int64_t row = first; row < p.M; row += step) {
        Row next;
        if (CH == 1 && row + step < p.M) load(next, row + step);
        float v[CH][8] = {}, h[8];
        if (p.y) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                settle8<FIT>(now.y[k], c + k * TH * 8, p.D);
                raw_to_float(now.y[k], v[k]);
            }
            norm_row<TH, FIT, CH>(p.post, p.post_eps, p.branch_scale, post, c, p.D, per_column, v, sum);
            if (p.gate) {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    float g[8];
                    settle8<FIT>(now.g[k], c + k * TH * 8, p.D);
                    raw_to_float(now.g[k], g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[k][i] *= g[i];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            settle8<FIT>(now.h[k], c + k * TH * 8, p.D);
            raw_to_float(now.h[k], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = fmaf(p.residual_scale, h[i], v[k][i]);
        }
        if (CH > 1 && TH < 1024 && row + step < p.M) load(next, row + step);
        if (p.h_out) {
#pragma unroll
            for (int k = 0; k < CH; ++k) store8(static_cast<H *>(p.h_out) + row * p.ldh_out + c + k * TH * 8, left(k), v[k]);
        }
        if (p.x || p.q) {
            norm_row<TH, FIT, CH>(p.pre, p.pre_eps, 1.0f, pre, c, p.D, per_column, v, sum);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int at = c + k * TH * 8;
                if (p.x) store8(static_cast<T *>(p.x) + row * p.ldx + at, left(k), v[k]);
                if (p.q) {
                    uint32_t a = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) a = max(a, abs_bits(v[k][i]));
                    float inverse;
                    const float s = fp8_scale(max16(a), &inverse);
                    store_codes(p.q + row * p.ldq + at, left(k), fp8_codes(v[k], inverse));
                    if ((threadIdx.x & 15) == 0 && left(k) > 0) p.scale[row * p.srow + (at >> 7) * p.scol] = s;
                }
            }
        }
        if (CH > 1 && TH == 1024 && row + step < p.M) load(next, row + step);
        now = next;
    }
}

// Rows too long for the registers: the fp32 row lies in LDS, where a thread reads back only what it wrote itself
// (4096 x 9001 fp32 111 us, 4.3 TB/s, bf16 88 us, 2.9; 1000 x 32768 bf16 113 us, one workgroup to a unit).
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
        if (w) raw_to_float(load8<CUT>(w, c, p.D), wv);
        if (b) raw_to_float(load8<CUT>(b, c, p.D), bv);
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
            long_row(p, lds, [&](int c, int, float (&v)[8]) { raw_to_float(load8<CUT>(static_cast<const T *>(p.y) + r * p.ldy, c, p.D), v); });
            norm_long_row(p, lds, p.post, p.post_eps, p.post_w, p.post_b, sum);
        }
        long_row(p, lds, [&](int c, int n, float (&v)[8]) {
            float h[8], g[8];
            raw_to_float(load8<CUT>(static_cast<const H *>(p.h) + r * p.ldh, c, p.D), h);
            if (p.gate) raw_to_float(load8<CUT>(gate, c, p.D), g);
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

template <typename T, typename H, int TH, int CH = 1>
static nq_status launch_norm(const NormParams &p, hipStream_t s)
{
    // up to sixteen waves to a compute unit (16384 x 4096 bf16 90 us; 8: 126, 24: 103)
    constexpr int ROWS = norm_rows(TH), WG = TH * ROWS;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(p.M, ROWS), 256 * (1024 / WG)));
    if constexpr (CH > 1) {
        k_block_norm<T, H, TH, CH, WHOLE><<<grid, WG, 0, s>>>(p);
    } else if (p.D == TH * 8) {
        k_block_norm<T, H, TH, CH, FULL><<<grid, WG, 0, s>>>(p);
    } else if (p.D % 8 == 0) {
        k_block_norm<T, H, TH, CH, WHOLE><<<grid, WG, 0, s>>>(p);
    } else {
        k_block_norm<T, H, TH, CH, CUT><<<grid, WG, 0, s>>>(p);
    }
    return launch_status();
}

template <typename T, typename H>
static nq_status norm_by_size(const NormParams &p, hipStream_t s)
{
    constexpr bool WIDE = sizeof(H) == 4;                   // the stream takes half of the registers
    const int chunks = (p.D + 7) / 8;
    if (p.M > 1024) {                                       // (few rows are faster with a wave each: 10 x 205 3.7 against 4.7 us)
        if (chunks <= 16) return launch_norm<T, H, 16>(p, s);
        if (chunks <= 32) return launch_norm<T, H, 32>(p, s);
    }
    if (chunks <= 64) return launch_norm<T, H, 64>(p, s);
    if (chunks <= 128) return launch_norm<T, H, 128>(p, s);
    if (chunks <= 256) return launch_norm<T, H, 256>(p, s);
    if (chunks <= 384) return launch_norm<T, H, 384>(p, s);
    if (chunks <= 512) return launch_norm<T, H, 512>(p, s);
    if (chunks <= 640) return launch_norm<T, H, 640>(p, s);
    // Sixteen columns to a thread make two workgroups to a unit of the one, 16384 x 8192 bf16 203 -> 184 us; with an fp32 stream
    // (8192 x 8192 fp32 195 -> 211 us) and with a cut-off chunk (16384 x 8190 bf16 215 -> 290) they cost more than that.
    if (p.D % 8 == 0) {
        if constexpr (!WIDE) {
            if (chunks <= 768) return launch_norm<T, H, 384, 2>(p, s);
            if (chunks <= 896) return launch_norm<T, H, 448, 2>(p, s);
            if (chunks <= 1024) return launch_norm<T, H, 512, 2>(p, s);
        }
        if (chunks > 1024 && chunks <= 1536) return launch_norm<T, H, 768, 2>(p, s);
        if constexpr (!WIDE) {
            if (chunks > 1536 && chunks <= 2048) return launch_norm<T, H, 1024, 2>(p, s);
        }
    }
    if (chunks <= 768) return launch_norm<T, H, 768>(p, s);
    if (chunks <= 1024) return launch_norm<T, H, 1024>(p, s);
    auto k = k_block_norm_long<T, H>;
    static std::atomic<uint64_t> granted{0};
    const nq_status st = grant_lds(k, NQ_NORM_MAX_D * 4, granted);
    if (st != NQ_OK) return st;
    k<<<(unsigned)std::min<int64_t>(p.M, 1 << 20), LONG_TH, chunks * 32, s>>>(p);
    return launch_status();
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
    if (j.dtype == NQ_DT_F32) return norm_by_size<float, float>(p, s);
    if (j.dtype == NQ_DT_F16) return j.h_dtype == NQ_DT_F16 ? norm_by_size<_Float16, _Float16>(p, s) : norm_by_size<_Float16, float>(p, s);
    return j.h_dtype == NQ_DT_BF16 ? norm_by_size<bf16_t, bf16_t>(p, s) : norm_by_size<bf16_t, float>(p, s);
}
