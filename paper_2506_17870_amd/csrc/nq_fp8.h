// Shared by the fp8 kernels (include/nq.h: nq_quantize_fp8, nq_gemm_fp8, nq_block_norm): element types, the e4m3 codes of
// eight values, host-side checks of a descriptor.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "nq_common.h"

namespace nq {

typedef _Float16 f8_h8 __attribute__((ext_vector_type(8)));
typedef float f8_f4 __attribute__((ext_vector_type(4)));

struct bf16_t {
    uint16_t bits;
};

// fp32 -> the type, rounded to nearest even (bf16 by the conversion instruction, two at a time)
typedef __bf16 f8_b2 __attribute__((ext_vector_type(2)));
typedef float f8_f2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f8_f2{a, b}, f8_b2));
}
__device__ __forceinline__ void from_float(float v, float *o) { *o = v; }
__device__ __forceinline__ void from_float(float v, _Float16 *o) { *o = (_Float16)v; }
__device__ __forceinline__ void from_float(float v, bf16_t *o) { o->bits = (uint16_t)pack_bf16(v, v); }

// Eight neighbouring elements as they lie in memory.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
    uint4 a, b;
};
template <>
struct Raw8<_Float16> {
    uint4 a;
};
template <>
struct Raw8<bf16_t> {
    uint4 a;
};

__device__ __forceinline__ void raw_to_float(const Raw8<float> &r, float (&v)[8])
{
    const uint32_t d[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, d[i]);
}
__device__ __forceinline__ void raw_to_float(const Raw8<_Float16> &r, float (&v)[8])
{
    const f8_h8 h = __builtin_bit_cast(f8_h8, r.a);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
}
__device__ __forceinline__ void raw_to_float(const Raw8<bf16_t> &r, float (&v)[8])
{
    const uint32_t d[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_bit_cast(float, d[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, d[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void float_to_raw(const float (&v)[8], Raw8<float> &r)
{
    r.a = __builtin_bit_cast(uint4, f8_f4{v[0], v[1], v[2], v[3]});
    r.b = __builtin_bit_cast(uint4, f8_f4{v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void float_to_raw(const float (&v)[8], Raw8<_Float16> &r)
{
    f8_h8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (_Float16)v[i];
    r.a = __builtin_bit_cast(uint4, h);
}
__device__ __forceinline__ void float_to_raw(const float (&v)[8], Raw8<bf16_t> &r)
{
    r.a = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Elements c .. c + 7 of a row of D, those past its end as zeros: fetch8() asks for them and settle8() puts them in their places, so
// that nothing waits before they are used.  The address need not be aligned to more than the type: the memory system takes wide
// accesses anywhere.  A chunk that the row's end cuts off is read as the row's last eight elements and moved down (one request,
// where a request per element would hold up the wave), in a row of fewer than eight by elements.
// FIT: CUT, any D; WHOLE, a multiple of eight, so that no chunk is cut off; FULL, every chunk is known to lie within the row.
enum Fit { CUT, WHOLE, FULL };
template <int FIT, typename T>
__device__ __forceinline__ Raw8<T> fetch8(const T *row, int c, int D)
{
    Raw8<T> r{};
    if (FIT != CUT) {
        if (FIT == FULL || c < D) __builtin_memcpy(&r, row + c, sizeof r);
    } else if (D >= 8) {
        if (c < D) __builtin_memcpy(&r, row + min(c, D - 8), sizeof r);
    } else if (c < D) {
        T e[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < D) e[i] = row[c + i];
        __builtin_memcpy(&r, e, sizeof r);
    }
    return r;
}
template <int FIT, typename T>
__device__ __forceinline__ void settle8(Raw8<T> &r, int c, int D)
{
    const int down = 8 - (D - c);
    if (FIT != CUT || down <= 0 || down >= 8 || D < 8) return;
    constexpr int W = (int)sizeof(r) / 4, PER = W / 8 ? 1 : 2;               // dwords; elements per dword
    uint32_t d[W];
    __builtin_memcpy(d, &r, sizeof r);
#pragma unroll
    for (int step = 4; step >= PER; step /= 2)
#pragma unroll
        for (int i = 0; i < W; ++i) d[i] = down & step ? (i + step / PER < W ? d[i + step / PER] : 0u) : d[i];
    if (PER == 2 && (down & 1)) {
#pragma unroll
        for (int i = 0; i < W; ++i) d[i] = __builtin_amdgcn_alignbit(i + 1 < W ? d[i + 1] : 0u, d[i], 16);
    }
    __builtin_memcpy(&r, d, sizeof r);
}
template <int FIT, typename T>
__device__ __forceinline__ Raw8<T> load8(const T *row, int c, int D)
{
    Raw8<T> r = fetch8<FIT>(row, c, D);
    settle8<FIT>(r, c, D);
    return r;
}
template <typename T>
__device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if (n >= 8) {
        Raw8<T> r;
        float_to_raw(v, r);
        __builtin_memcpy(p, &r, sizeof r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) from_float(v[i], p + i);
    }
}

// The scale of a block with largest magnitude a (its bits, so that a NaN, the largest pattern of all, wins every maximum),
// and the factor of its codes.  Both quotients are the correctly rounded ones: an approximation good to a unit, and a step with the
// remainder, which a fused multiply-add gives exactly (Markstein 1990); a compiler's division also scales for operands that
// cannot occur here (s is between 2^-126 and 2^120), and there is one for every eight elements.
__device__ __forceinline__ float fp8_scale(uint32_t a_bits, float *inverse)
{
    const float a = __builtin_bit_cast(float, a_bits), c = 1.0f / 448.0f;
    float s = a * c;
    s = fmaf(fmaf(-448.0f, s, a), c, s);
    s = s < 0x1p-126f ? 0x1p-126f : s;
    s = a_bits == 0 ? 1.0f : s;
    float y = __builtin_amdgcn_rcpf(s);
    y = fmaf(fmaf(-s, y, 1.0f), y, y);
    y = fmaf(fmaf(-s, y, 1.0f), y, y);
    const bool finite = a_bits < 0x7f800000u;
    *inverse = finite ? y : a_bits == 0x7f800000u ? 0.0f : a;             // 1 / infinity, 1 / NaN
    return finite ? s : a;
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// Codes of eight values.  |v * inverse| <= 448 (1 + 2^-22) in a block with finite values, which rounds to 448 at most, so no
// clamp is needed; NaN becomes the NaN code.
__device__ __forceinline__ uint2 fp8_codes(const float (&v)[8], float inverse)
{
    uint32_t d[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inverse, v[4 * i + 1] * inverse, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inverse, v[4 * i + 3] * inverse, w, true);
        d[i] = (uint32_t)w;
    }
    return make_uint2(d[0], d[1]);
}
__device__ __forceinline__ void store_codes(uint8_t *p, int n, uint2 c)
{
    if (n >= 8) {
        __builtin_memcpy(p, &c, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (uint8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
    }
}

// Reductions over sixteen neighbouring lanes by data-parallel moves: neighbours, pairs, halves of eight, halves of sixteen.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, v))); }

__device__ __forceinline__ uint32_t max16(uint32_t v)
{
    v = max(v, dpp<0xB1>(v));
    v = max(v, dpp<0x4E>(v));
    v = max(v, dpp<0x141>(v));
    return max(v, dpp<0x140>(v));
}
__device__ __forceinline__ float sum16(float v)
{
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    return v + dpp<0x140>(v);
}
// ... and over the wave's 64, the same value in every lane.
__device__ __forceinline__ float sum64(float v)
{
    const int r = __builtin_bit_cast(int, sum16(v));
    auto row = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(r, lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}

// 1 / sqrt(x), the hardware's (good to a unit) also where x is too small for it (a denormal, which it takes for 0).
__device__ __forceinline__ float inverse_root(float x)
{
    const bool small = x < 0x1p-100f;
    const float r = __builtin_amdgcn_rsqf(small ? x * 0x1p80f : x);
    return small ? r * 0x1p40f : r;
}

// ---- host ------------------------------------------------------------------------------------------------------

inline int dtype_bytes(int dtype) { return dtype == NQ_DT_F32 ? 4 : 2; }
inline bool is_dtype(int dtype) { return dtype == NQ_DT_F32 || dtype == NQ_DT_F16 || dtype == NQ_DT_BF16; }
inline bool aligned_to(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// rows * ld elements stay far inside 64 bits for every size that is let through
constexpr int64_t FP8_MAX_ROWS = int64_t(1) << 40, FP8_MAX_LD = int64_t(1) << 20;

inline nq_status check_fp8(const nq_fp8 *q)
{
    if (!q || q->rows < 0 || q->cols < 0 || q->scale_row_step < 0 || q->scale_col_step < 0) return NQ_ERR_INVALID_ARG;
    if (q->block_rows != 1 && q->block_rows != 128) return NQ_ERR_INVALID_ARG;
    if (q->cols > NQ_MAX_K || q->rows > FP8_MAX_ROWS || q->ld < q->cols || q->ld > FP8_MAX_LD) return NQ_ERR_SHAPE;
    if (q->scale_row_step > FP8_MAX_LD || q->scale_col_step > FP8_MAX_ROWS) return NQ_ERR_SHAPE;
    if (q->rows == 0 || q->cols == 0) return NQ_OK;
    if (!q->d_q || !q->d_scale) return NQ_ERR_INVALID_ARG;
    return aligned_to(q->d_scale, 4) ? NQ_OK : NQ_ERR_ALIGN;
}

// A [rows][cols] operand of `dtype`, rows ld elements apart.
inline nq_status check_matrix(const void *p, int dtype, int64_t cols, int64_t ld)
{
    if (!p) return NQ_ERR_INVALID_ARG;
    if (ld < cols || ld > (int64_t(1) << 32)) return NQ_ERR_SHAPE;
    return aligned_to(p, dtype_bytes(dtype)) ? NQ_OK : NQ_ERR_ALIGN;
}

// Grants a kernel `bytes` of dynamic LDS, more than the 64 KB that every kernel has: once on each device, whose copy of the kernel
// it is that has the limit (`devices`: those done, a static of the caller's for each kernel).  A refusal is reported, and the next call asks
// again.  `bytes` is the most that the kernel is ever launched with, so that no call lowers the limit under another.
template <typename K>
nq_status grant_lds(K kernel, int bytes, std::atomic<uint64_t> &devices)
{
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return NQ_ERR_HIP;
    }
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (devices.load(std::memory_order_acquire) & bit) return NQ_OK;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) {
        (void)hipGetLastError();
        return NQ_ERR_HIP;
    }
    devices.fetch_or(bit, std::memory_order_release);
    return NQ_OK;
}

// n / d == (n * m) >> (32 + s) for every n < 2^31 and 1 <= d < 2^31, m and s made here (m fits 32 bits: 2^(32+s) / d with
// 2^s <= d < 2^(s+1) lies in (2^31, 2^32]; rounded up it is off by less than one part in 2^31 / n).  d = 1 gives m = 2^32,
// kept as 0 and taken apart in divide().
struct Divider {
    uint32_t d, m;
    int s;
};
inline Divider make_divider(uint32_t d)
{
    int s = 0;
    while ((d >> (s + 1)) != 0) ++s;
    if ((d & (d - 1)) == 0) return Divider{d, 0, s};     // a power of two: a shift
    return Divider{d, (uint32_t)(((uint64_t(1) << (32 + s)) + d - 1) / d), s};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divider &v) { return v.m ? __umulhi(n, v.m) >> v.s : n >> v.s; }

}  // namespace nq
