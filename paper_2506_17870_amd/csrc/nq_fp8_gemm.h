// The e4m3 matrix product with block scales: what its kernels share.
//
//   Y[m][n] = sum_b sx[m][b] * sw[n / 128][b] * P_b[m][n] + bias[n],   P_b = sum over block b's 128 columns of x[m][k] * w[n][k]
//
// One v_mfma_f32_16x16x128_f8f6f4 makes P_b of 16 weight rows and 16 tokens.  The weights are its A operand and the
// tokens its B operand, so that in the result a lane holds one token (lane % 16) and four neighbouring outputs
// 4 * (lane / 16) + i: the token's scale is one value per lane and the weights' scale one per wave, a single factor for the
// lane's four sums, and the four outputs are stored side by side.  The products of a block start from zero and are added
// to the running sums with four fused multiply-adds in fp32, as the formula says.  (The matrix core can scale its operands
// itself, but by powers of two only.)  A lane of either operand holds 32 bytes of a row; which of the block's columns they
// are does not matter as long as both operands agree, so a lane takes the 16-byte pieces lane / 16 and 4 + lane / 16.
#pragma once
#include <hip/hip_ext.h>

#include "nq_fp8.h"

namespace nq {

typedef int f8_v8i __attribute__((ext_vector_type(8)));
typedef int f8_v4i __attribute__((ext_vector_type(4)));

struct Fp8GemmParams {
    const uint8_t *x, *w;
    const float *sx, *sw, *bias;
    void *y;
    int64_t ldx, ldw, ldy, sxr, sxc, swr, swc;
    int M, N, K, KB;                       // KB: column blocks
    int sx_span;                           // bytes from the first scale of a tile's tokens to past the last (tiled kernel)
};

__device__ __forceinline__ f8_v8i fp8_frag(f8_v4i lo, f8_v4i hi)
{
    return f8_v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// A lane's 32 codes of a block as the matrix core takes them.
//
// WIDE = false: the codes themselves.  The fp8 matrix instructions (all of them, measured) put products that lie close together
// on the exponent of the largest and cut them off about 14 bits below it before they add them in fp32: 1.4e-5 of the result
// (2-norm) for normal codes, 5e-5 for codes of every size alike.  That is a fifteenth of what rounding the result to f16 costs
// and a hundredth of bf16's, so 16-bit outputs are made with it.
// WIDE = true, for fp32 outputs, whose own rounding would be a thousand times smaller: every code is exactly an f16 number and
// every product of two exactly an fp32 one; the f16 instruction cuts nothing off (1e-8 on the same codes).  It has half the
// rate, and a conversion for every two codes comes before it.
typedef _Float16 f8_h2 __attribute__((ext_vector_type(2)));
template <bool WIDE>
struct Fp8Operand {
    f8_v8i v;
    __device__ __forceinline__ void set(f8_v8i codes) { v = codes; }
};
template <>
struct Fp8Operand<true> {
    f8_h8 v[4];
    __device__ __forceinline__ void set(f8_v8i codes)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f8_h2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[i], 1.0f, false);
            const f8_h2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[i], 1.0f, true);
            const int at = 4 * (i & 1);
            v[i >> 1][at] = lo[0];
            v[i >> 1][at + 1] = lo[1];
            v[i >> 1][at + 2] = hi[0];
            v[i >> 1][at + 3] = hi[1];
        }
    }
};

// P of one block.  (both scale operands 0: the instruction without scales)
__device__ __forceinline__ f8_f4 fp8_mfma(const Fp8Operand<false> &w, const Fp8Operand<false> &x)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, f8_f4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f8_f4 fp8_mfma(const Fp8Operand<true> &w, const Fp8Operand<true> &x)
{
    f8_f4 r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) r = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[i], x.v[i], r, 0, 0, 0);
    return r;
}
__device__ __forceinline__ void fp8_add(f8_f4 &acc, f8_f4 p, float s)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(p[i], s, acc[i]);
}

// The biases of a lane's outputs n + 16 j + 4 (lane / 16) + 0 .. 3.
template <int TN>
__device__ __forceinline__ void fp8_bias(const Fp8GemmParams &p, int n, int lane, f8_f4 (&b)[TN])
{
    if (!p.bias) return;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int at = n + j * 16 + 4 * (lane >> 4);
        b[j] = f8_f4{0.0f, 0.0f, 0.0f, 0.0f};
        if (at + 4 <= p.N) {
            __builtin_memcpy(&b[j], p.bias + at, 16);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (at + q < p.N) b[j][q] = p.bias[at + q];
        }
    }
}

// A wave's 16 * TM tokens x 16 * TN outputs from token m and output n on.  The matrix core leaves a token's outputs in pieces of
// four per lane: stored like that a wave's store would touch sixteen rows with 32 bytes each (a tile of 256 x 256 took 12 us).  They go
// through LDS instead, `mine` being 16 * TM * TN * 16 elements that no other wave uses, and leave as whole rows, 16 bytes per lane at
// any alignment (2773 x 2474 x 554, whose rows start on four bytes, 12.1 us; element by element 21.4).
// The 16-byte units of a row lie exchanged so that sixteen rows' equal units, which one write covers, lie in different banks.
// `bias`: those of the lane's outputs, from fp8_bias().
template <typename T, int TN, int TM>
__device__ __forceinline__ void fp8_store_tile(const Fp8GemmParams &p, int m, int n, f8_f4 (&acc)[TM][TN], const f8_f4 (&bias)[TN], uint8_t *mine,
                                               int lane)
{
    const int r16 = lane & 15, g4 = lane >> 4;
    constexpr int ROW = TN * 16 * (int)sizeof(T), UNITS = ROW / 16, E = 16 / (int)sizeof(T);
    constexpr int MASK = UNITS < 16 ? UNITS - 1 : 15, SHARE = UNITS < 16 ? 16 / UNITS : 1;      // rows that lie once round the banks
    auto place = [](int row, int unit) { return row * ROW + 16 * (unit ^ ((row / SHARE) & MASK)); };
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const f8_f4 v = p.bias ? acc[i][j] + bias[j] : acc[i][j];
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<f8_f4 *>(mine + place(i * 16 + r16, j * 4 + g4)) = v;
            } else {
                T o[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) from_float(v[q], o + q);
                *reinterpret_cast<uint2 *>(mine + place(i * 16 + r16, j * 2 + (g4 >> 1)) + 8 * (g4 & 1)) = __builtin_bit_cast(uint2, o);
            }
        }
    }
    // (the hardware keeps a wave's writes and reads of LDS in order; the compiler, which sees other types in them, has to be told)
    asm volatile("" ::: "memory");
    constexpr int AT_ONCE = 64 / UNITS;                    // rows of a store
    const int unit = lane % UNITS, col = n + unit * E;
#pragma unroll
    for (int i = 0; i < (16 * TM + AT_ONCE - 1) / AT_ONCE; ++i) {
        const int row = i * AT_ONCE + lane / UNITS;
        if (16 * TM < AT_ONCE && row >= 16 * TM) return;
        const uint4 v = *reinterpret_cast<const uint4 *>(mine + place(row, unit));
        if (m + row >= p.M || col >= p.N) continue;
        T *y = static_cast<T *>(p.y) + (int64_t)(m + row) * p.ldy + col;
        if (col + E <= p.N) {
            __builtin_memcpy(y, &v, 16);
        } else {
            T e[E];
            __builtin_memcpy(e, &v, 16);
#pragma unroll
            for (int q = 0; q < E; ++q)
                if (col + q < p.N) y[q] = e[q];
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

// nq_gemm.hip: the events of nq_profile_next_launch, which are taken by this, and what nq_profile_last_kernel reports.
void take_profile_events(void **start, void **stop);
void note_last_kernel(int family, int variant);
constexpr int FP8_FAMILY = 12, FP8_ANY = 100;            // variants: the tile form, or FP8_ANY + groups for rows on any byte

struct Fp8Launch {
    hipStream_t stream;
    void *start, *stop;                                  // events of this launch, or null
};
template <typename K>
nq_status launch_fp8(const Fp8Launch &at, K kernel, int64_t tiles, int threads, int lds, const Fp8GemmParams &p)
{
    if (at.start || at.stop)
        hipExtLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(threads), (uint32_t)lds, at.stream, (hipEvent_t)at.start, (hipEvent_t)at.stop, 0, p);
    else
        kernel<<<(unsigned)tiles, threads, lds, at.stream>>>(p);
    return launch_status();
}

}  // namespace nq
