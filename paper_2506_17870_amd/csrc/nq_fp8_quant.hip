// nq_quantize_fp8: floats -> e4m3 codes with a scale for each block of 128 columns, behind an activation function and a product.
// Bound by the bytes: each input is read once and each code written once, and the block's values stay in registers between
// the maximum and the codes.
#include "nq_fp8.h"

namespace nq {

struct QuantParams {
    const void *x, *mul;
    uint8_t *q;
    float *scale;
    int64_t ldx, ldmul, ldq, srow, scol, row0;
    uint32_t rows, groups;                 // rows of this launch; rows * column blocks
    int K;
    Divider by_blocks;                     // column blocks of a row
};

// Exponentials and quotients are the hardware's base-2 exponential and reciprocal, each good to a unit.  What the steps make of that is said
// at each function, in parts of its result; a code's step is 2^-4 of its value at the least, so one in a million or two moves.
template <int ACT>
__device__ __forceinline__ float activate(float v)
{
    if constexpr (ACT == NQ_ACT_RELU) return v < 0.0f ? 0.0f : v;             // (NaN stays)
    // v / (1 + exp(-v)), for negative v as v exp(v) / (1 + exp(v)), whose parts stay between 0 and 2.  exp(-|v|) is the square of p = exp2(x),
    // x = -|v| / (2 ln 2) rounded to fp32, so that it reaches below the normal numbers, times 1 + d, d being what the rounding took from
    // the exponent (an exponent of 126 left as rounded costs the result 24 parts in 2^23).  Off by 8 parts in 2^23 at most
    // (exponential, twice, reciprocal, four products, a sum), 64 below -87, where exp(v) is subnormal.  4096 x 4096 bf16 12.1 us, as
    // v / (1 + exp2(-v / ln 2)) without either 10.8; in a gated layer (below) the bytes hide the difference.
    if constexpr (ACT == NQ_ACT_SILU) {
        const float z = fabsf(v), x = z * -0.721347511f, p = __builtin_amdgcn_exp2f(x), d = fmaf(x, -1.38629436f, -z);
        const float w = fminf(fmaxf(fmaf(p * p, d, p * p), 0.0f), 1.0f);      // (no NaN for an infinite v; free: the clamp of the instruction)
        const float r = v * __builtin_amdgcn_rcpf(1.0f + w);
        return r * (v < 0.0f ? w : 1.0f);
    }
    // The tail of the normal distribution is exp(-v^2 / 2) times a polynomial of 1 / (1 + 0.3 |v|) with the least largest relative error
    // (1.5e-7 over 0 <= |v| <= 14; fitted here), so that nothing cancels for negative v.  Off by 8 parts in 2^23 for positive v, by 8 + 0.6 v^2
    // for negative (the exponent is rounded to fp32 twice: 23 parts at -5, 100 at -12); the textbook form v (1 + erf) / 2 in fp32
    // loses everything below -5.  Results below 2^-126 come out as 0.  The library's erf takes three times the instructions and bound
    // the kernel (1009 x 5003 f16 8.0 us).
    if constexpr (ACT == NQ_ACT_GELU) {
        const float z = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(0.3f, z, 1.0f));
        float q = fmaf(t, 0.035674829f, -0.157203302f);
        q = fmaf(t, q, 0.206353873f);
        q = fmaf(t, q, -0.0536839664f);
        q = fmaf(t, q, 0.12856178f);
        q = fmaf(t, q, 0.0999134481f);
        q = fmaf(t, q, 0.120753966f);
        q = fmaf(t, q, 0.119629301f) * t;
        const float tail = q * __builtin_amdgcn_exp2f(v * v * -0.72134752f);
        // (infinity times nothing is no tail)
        return v >= 0.0f ? (tail == 0.0f ? v : fmaf(-v, tail, v)) : v * tail;
    }
    // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), u = sqrt(2 / pi) (v + 0.044715 v^3), as SiLU with p = exp(-|u|) (2^-72 at v = -10.5, whose
    // square the reciprocal would not take).  Off by 8 parts in 2^23, and 1.2 for each unit of the exponent 2.3 |v| + 0.103 |v|^3, which is
    // rounded to fp32 four times; the function itself is off by more than that from what it stands for.  4096 x 4096 bf16 12.5 us.
    if constexpr (ACT == NQ_ACT_GELU_TANH) {
        const float p = __builtin_amdgcn_exp2f(fabsf(v) * fmaf(v * v, -0.0514716208f, -1.15110409f));
        const float r = v * __builtin_amdgcn_rcpf(fmaf(p, p, 1.0f)), k = v < 0.0f ? p : 1.0f;
        return r * k * k;
    }
    return v;
}

template <int ACT, typename T>
__device__ __forceinline__ uint32_t act_and_max(const Raw8<T> &x, const Raw8<T> *m, float (&v)[8])
{
    raw_to_float(x, v);
    float u[8];
    if (m) raw_to_float(*m, u);
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = activate<ACT>(v[i]);
        if (m) v[i] *= u[i];
        a = max(a, abs_bits(v[i]));
    }
    return a;
}

// A scale for each 1 x 128: eight columns per thread, sixteen threads per block of columns (16384 x 8192 bf16 SiLU times a second
// matrix 113 us, 6.0 TB/s of operands in part cached; GELU in 16 bits is bound by the vector unit, 4096 x 4096 16 us).
template <typename T, int ACT, bool MUL>
__global__ void __launch_bounds__(256) k_fp8_rows(const QuantParams p)
{
    const uint32_t group = blockIdx.x * 16u + (threadIdx.x >> 4);
    if (group >= p.groups) return;
    const uint32_t r = divide(group, p.by_blocks), b = group - r * p.by_blocks.d;
    const int64_t row = p.row0 + r;
    const int c = (int)b * 128 + (threadIdx.x & 15) * 8;
    const int n = min(8, max(0, p.K - c));
    const Raw8<T> x = load8<CUT>(static_cast<const T *>(p.x) + row * p.ldx, c, p.K);
    Raw8<T> m{};
    if constexpr (MUL) m = load8<CUT>(static_cast<const T *>(p.mul) + row * p.ldmul, c, p.K);
    float v[8], inverse;
    const uint32_t a = max16(act_and_max<ACT>(x, MUL ? &m : nullptr, v));
    const float s = fp8_scale(a, &inverse);
    store_codes(p.q + row * p.ldq + c, n, fp8_codes(v, inverse));
    if ((threadIdx.x & 15) == 0) p.scale[row * p.srow + b * p.scol] = s;
}

// A scale for each 128 x 128: a workgroup per block, eight columns of every TH / 16-th row per thread.
template <typename T, int ACT, bool MUL, int TH>
__global__ void __launch_bounds__(TH) k_fp8_tiles(const QuantParams p)
{
    constexpr int STEP = TH / 16, ROWS = 128 / STEP;
    __shared__ uint32_t largest[TH / 64];
    const uint32_t rb = divide(blockIdx.x, p.by_blocks), b = blockIdx.x - rb * p.by_blocks.d;
    const int c = (int)b * 128 + (threadIdx.x & 15) * 8;
    const int n = min(8, max(0, p.K - c));
    const uint32_t r0 = rb * 128 + (threadIdx.x >> 4);
    Raw8<T> x[ROWS], m[MUL ? ROWS : 1];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = p.row0 + r0 + STEP * i;
        const int here = r0 + STEP * i < p.rows ? p.K : 0;   // (a row that is not there: no elements)
        x[i] = fetch8<CUT>(static_cast<const T *>(p.x) + row * p.ldx, c, here);
        if constexpr (MUL) m[i] = fetch8<CUT>(static_cast<const T *>(p.mul) + row * p.ldmul, c, here);
    }
    uint32_t a = 0;
    float v[8], inverse;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        settle8<CUT>(x[i], c, p.K);
        if constexpr (MUL) settle8<CUT>(m[i], c, p.K);
        a = max(a, act_and_max<ACT>(x[i], MUL ? &m[i] : nullptr, v));
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) a = max(a, (uint32_t)__shfl_xor((int)a, k));
    if ((threadIdx.x & 63) == 0) largest[threadIdx.x >> 6] = a;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TH / 64; ++i) a = max(a, largest[i]);
    const float s = fp8_scale(a, &inverse);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = p.row0 + r0 + STEP * i;
        const int here = r0 + STEP * i < p.rows ? n : 0;
        act_and_max<ACT>(x[i], MUL ? &m[i] : nullptr, v);
        store_codes(p.q + row * p.ldq + c, here, fp8_codes(v, inverse));
    }
    if (threadIdx.x == 0) p.scale[(p.row0 / 128 + rb) * p.srow + b * p.scol] = s;
}

template <typename T, int ACT, bool MUL>
static void launch_quant(const QuantParams &p, int block_rows, hipStream_t s)
{
    if (block_rows == 1) {
        const dim3 grid((p.groups + 15) / 16);
        k_fp8_rows<T, ACT, MUL><<<grid, 256, 0, s>>>(p);
    } else {
        const dim3 grid((p.rows + 127) / 128 * p.by_blocks.d);
        // 1024 threads where a compute unit has one block (423 x 6912 bf16 3.8 us, with 512 3.9, with 256 4.9) and for fp32
        // (8192 x 8192 57 us, 60, 63); 512 else (1892 x 2476 bf16 6.2 us, with 1024 6.3, with 256 7.5).
        if (sizeof(T) == 4 || grid.x <= 256)
            k_fp8_tiles<T, ACT, MUL, 1024><<<grid, 1024, 0, s>>>(p);
        else if constexpr (sizeof(T) == 2)
            k_fp8_tiles<T, ACT, MUL, 512><<<grid, 512, 0, s>>>(p);
    }
}

template <typename T>
static void launch_act(const QuantParams &p, int act, int block_rows, hipStream_t s)
{
#define NQ_QUANT_ACT(A)                                                   \
    case A:                                                               \
        if (p.mul)                                                        \
            launch_quant<T, A, true>(p, block_rows, s);              \
        else                                                              \
            launch_quant<T, A, false>(p, block_rows, s);             \
        break;
    switch (act) {
        NQ_QUANT_ACT(NQ_ACT_NONE)
        NQ_QUANT_ACT(NQ_ACT_RELU)
        NQ_QUANT_ACT(NQ_ACT_SILU)
        NQ_QUANT_ACT(NQ_ACT_GELU)
        NQ_QUANT_ACT(NQ_ACT_GELU_TANH)
    default: break;
    }
#undef NQ_QUANT_ACT
}

}  // namespace nq

using namespace nq;

extern "C" nq_status nq_quantize_fp8(const void *d_x, int dtype, int64_t ldx, const void *d_mul, int64_t ldmul, int act,
                                     const nq_fp8 *q, void *stream)
{
    if (!is_dtype(dtype) || act < NQ_ACT_NONE || act > NQ_ACT_GELU_TANH) return NQ_ERR_INVALID_ARG;
    nq_status st = check_fp8(q);
    if (st != NQ_OK) return st;
    if (q->rows == 0 || q->cols == 0) return NQ_OK;
    if ((st = check_matrix(d_x, dtype, q->cols, ldx)) != NQ_OK) return st;
    if (d_mul && (st = check_matrix(d_mul, dtype, q->cols, ldmul)) != NQ_OK) return st;

    QuantParams p;
    p.x = d_x;
    p.mul = d_mul;
    p.q = q->d_q;
    p.scale = q->d_scale;
    p.ldx = ldx;
    p.ldmul = ldmul;
    p.ldq = q->ld;
    p.srow = q->scale_row_step;
    p.scol = q->scale_col_step;
    p.K = (int)q->cols;
    const uint32_t blocks = (uint32_t)ceil_div(q->cols, 128);
    p.by_blocks = make_divider(blocks);
    // A dispatch has fewer than 2^32 threads: at most 2^27 blocks of columns with sixteen (with 128 rows each: eight) threads to one,
    // whole blocks of 128 rows.
    const int64_t step = std::max<int64_t>(128, (int64_t(1) << 27) / blocks / 128 * 128);
    for (p.row0 = 0; p.row0 < q->rows; p.row0 += step) {
        p.rows = (uint32_t)std::min(step, q->rows - p.row0);
        p.groups = p.rows * blocks;
        if (dtype == NQ_DT_F32)
            launch_act<float>(p, act, q->block_rows, (hipStream_t)stream);
        else if (dtype == NQ_DT_F16)
            launch_act<_Float16>(p, act, q->block_rows, (hipStream_t)stream);
        else
            launch_act<bf16_t>(p, act, q->block_rows, (hipStream_t)stream);
        if ((st = launch_status()) != NQ_OK) return st;
    }
    return NQ_OK;
}
