// nq_gemm_fp8: the kernels and the choice between them.  nq_fp8_gemm.h has the mathematics.
#include "nq_fp8_gemm_tile.h"

namespace nq {

// ---- any alignment ---------------------------------------------------------------------------------------------
// Rows that start on any byte: the direct loads of the tiles want them on 16, ordinary ones do not.  A piece of 16 bytes that the row's
// end cuts off is read as the row's last 16 and moved down by any_settle(); rows of fewer than 16 bytes go by bytes.
__device__ __forceinline__ f8_v4i any_fetch(const uint8_t *row, int k, int K)
{
    f8_v4i r = {0, 0, 0, 0};
    if (k >= K) return r;
    if (K >= 16) {
        __builtin_memcpy(&r, row + min(k, K - 16), 16);
    } else {
        uint32_t d[4] = {};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < K) d[i >> 2] |= (uint32_t)row[i] << (8 * (i & 3));
        __builtin_memcpy(&r, d, 16);
    }
    return r;
}
__device__ __forceinline__ void any_settle(f8_v4i &r, int k, int K)
{
    const int down = 16 - (K - k);                         // bytes
    if (down <= 0 || down >= 16 || K < 16) return;
    uint32_t d[4];
    __builtin_memcpy(d, &r, 16);
#pragma unroll
    for (int step = 2; step >= 1; step /= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = (down >> 2) & step ? (i + step < 4 ? d[i + step] : 0u) : d[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = __builtin_amdgcn_alignbyte(i + 1 < 4 ? d[i + 1] : 0u, d[i], down & 3);
    __builtin_memcpy(&r, d, 16);
}

// Tile of 64 weight rows x 64 tokens, G groups of four waves of 32 x 32; group g takes the column blocks g, g + G, ... through LDS
// of its own, the next block's pieces on their way in registers while one is worked on, and the groups' sums are added in order.
// A row's eight 16-byte pieces lie exchanged, piece c at c ^ ((row / 2) & 7): two rows are once round the 64 banks, and sixteen rows'
// pieces c in sixteen different places.  Bound by the loads' latency
// and by placing what they bring: 16 x 4096 x 4096 17 us, 1024 x 4096 x 4096 68, 4096^3 186, where rows on 16 bytes take 5, 24 and
// 62; put together from aligned dwords, without the next block ahead and in one group these took 51, 142 and 417.
template <typename T, int G>
__global__ void __launch_bounds__(256 * G) k_fp8_gemm_any(const Fp8GemmParams p)
{
    __shared__ f8_v4i lds[G][2][64 * 8];                   // weights, tokens
    const int group = G == 1 ? 0 : threadIdx.x >> 8, id0 = threadIdx.x & 255;
    const int nblocks = (p.N + 63) / 64;
    const int bm = blockIdx.x / nblocks, bn = blockIdx.x - bm * nblocks;
    const int m0 = bm * 64, n0 = bn * 64;
    const int lane = threadIdx.x & 63, wave = id0 >> 6;
    const int wn = (wave & 1) * 32, wm = (wave >> 1) * 32;
    const int r16 = lane & 15, g = lane >> 4;
    auto &panel = lds[group];
    const float *sw = p.sw + (int64_t)(min(n0 + wn, p.N - 1) >> 7) * p.swr;

    f8_v4i piece[4];                                       // two of the weights, two of the tokens
    float scale[3];                                        // of the lane's tokens and of the weights
    auto fetch = [&](int kb) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int id = (i & 1) * 256 + id0, row = id >> 3, k = kb * 128 + (id & 7) * 16;
            const int at = (i >= 2 ? m0 : n0) + row;
            const bool there = kb < p.KB && at < (i >= 2 ? p.M : p.N);
            piece[i] = any_fetch(i >= 2 ? p.x + (int64_t)at * p.ldx : p.w + (int64_t)at * p.ldw, there ? k : p.K, p.K);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = m0 + wm + i * 16 + r16;
            scale[i] = kb < p.KB && m < p.M ? p.sx[(int64_t)m * p.sxr + (int64_t)kb * p.sxc] : 0.0f;
        }
        scale[2] = kb < p.KB ? sw[(int64_t)kb * p.swc] : 0.0f;
    };
    f8_f4 acc[2][2] = {};
    fetch(group);
    for (int kb = group; kb - group < p.KB; kb += G) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int id = (i & 1) * 256 + id0, row = id >> 3, c = id & 7;
            any_settle(piece[i], kb * 128 + c * 16, p.K);
            panel[i >> 1][row * 8 + (c ^ ((row >> 1) & 7))] = piece[i];
        }
        const float s[2] = {scale[0] * scale[2], scale[1] * scale[2]};
        __syncthreads();
        fetch(kb + G);
        auto frag = [&](int which, int row) {
            const f8_v4i *q = panel[which] + row * 8;
            const int e = (row >> 1) & 7;
            Fp8Operand<sizeof(T) == 4> o;
            o.set(fp8_frag(q[g ^ e], q[(g + 4) ^ e]));
            return o;
        };
        const auto w0 = frag(0, wn + r16), w1 = frag(0, wn + 16 + r16);
#pragma unroll
        for (int tm = 0; tm < 2; ++tm) {
            const auto x = frag(1, wm + tm * 16 + r16);
            fp8_add(acc[tm][0], fp8_mfma(w0, x), s[tm]);
            fp8_add(acc[tm][1], fp8_mfma(w1, x), s[tm]);
        }
    }
    __syncthreads();
    if constexpr (G > 1) {
        f8_f4 *sum = reinterpret_cast<f8_f4 *>(lds);
        if (group > 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[((group - 1) * 4 + i) * 256 + id0] = acc[i >> 1][i & 1];
        __syncthreads();
        if (group > 0) return;
        for (int h = 1; h < G; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] += sum[((h - 1) * 4 + i) * 256 + id0];
    }
    f8_f4 bias[2];
    fp8_bias(p, n0 + wn, lane, bias);
    // (the last group's part of the memory holds no sums)
    fp8_store_tile<T, 2, 2>(p, m0 + wm, n0 + wn, acc, bias, reinterpret_cast<uint8_t *>(lds[G - 1]) + wave * (32 * 32 * (int)sizeof(T)), lane);
}

template <typename T>
static nq_status launch_any(const Fp8GemmParams &p, const Fp8Launch &s)
{
    const int64_t tiles = ceil_div(p.M, 64) * ceil_div(p.N, 64);
    const bool few = tiles <= 512;                         // two to a compute unit
    note_last_kernel(FP8_FAMILY, FP8_ANY + (few ? 4 : 1));
    return few ? launch_fp8(s, k_fp8_gemm_any<T, 4>, tiles, 1024, 0, p) : launch_fp8(s, k_fp8_gemm_any<T, 1>, tiles, 256, 0, p);
}

// ---- which tile ------------------------------------------------------------------------------------------------
// What a tile form takes, in microseconds, fitted to launches of 193 (fp32 outputs: 77) random sizes from 1 x 100 x 100 to 8192^3:
// start + a round of tiles, `occ` to a compute unit, for each 256 * occ of them: per_tile + it * per_step, either with a part
// that grows with the round's share of occupied units; it: steps of G column blocks.  The form with the least is taken: on those
// sizes 0.8 % (0.4 %) slower than the fastest of 17 forms timed for each, 9 % at worst.
struct Fp8Form {
    int BN, BM, G, occ;
    float start, tile, tile_full, step, step_full;
};

static double form_time(const Fp8Form &f, int M, int N, int KB)
{
    const int64_t tiles = ceil_div(M, f.BM) * ceil_div(N, f.BN), slots = 256 * f.occ, rounds = tiles / slots, rest = tiles % slots;
    const double it = (double)ceil_div(KB, f.G);
    auto round = [&](double load) { return f.tile + f.tile_full * load + it * (f.step + f.step_full * load); };
    // (the last round's load: half of it what the tiles share over the card, half what the fullest compute unit has)
    const double load = 0.5 * ((double)rest / slots + (double)ceil_div(rest, 256) / f.occ);
    return f.start + rounds * round(1.0) + (rest ? round(load) : 0.0);
}

// Few tokens: small tiles with many waves along the columns: the weights stream (24 x 8192 x 8192 12.6 us, 5.4 TB/s), and up to 256 tiles
// three stages have a unit's weights on their way at once (1 x 4096 x 4096 5.0 us, with two stages 5.8).  Some hundred: the largest tile of which there are still 256.  Many: tiles of 256 x 256 (16-bit outputs, 8192^3
// 2.36 PFLOP/s; the register-only stream of these instructions and multiply-adds reaches 3.5 on such data, the same kernel without
// its loads 2.7); fp32 outputs need the registers for their wider operands and stay at 128 x 128.
static const Fp8Form FORMS_16[] = {
    {16, 16, 4, 4, 2.15f, 0.00f, 1.33f, 0.218f, 0.439f},   {16, 16, 8, 1, 1.51f, 0.53f, 1.16f, 0.312f, 0.073f},
    {64, 16, 4, 1, 1.58f, 0.68f, 1.16f, 0.414f, 0.102f},   {64, 32, 4, 1, 1.64f, 0.97f, 1.70f, 0.492f, 0.137f},
    {64, 64, 2, 2, 2.01f, 0.00f, 2.15f, 0.408f, 0.461f},   {128, 128, 1, 2, 2.52f, 0.00f, 4.27f, 0.394f, 0.669f},
    {64, 64, 2, 1, 1.43f, 0.79f, 1.36f, 0.396f, 0.081f},   {128, 128, 1, 1, 1.34f, 0.88f, 2.73f, 0.348f, 0.236f},
    {256, 128, 1, 1, 1.88f, 0.00f, 5.52f, 0.450f, 0.539f}, {256, 256, 1, 1, 0.86f, 0.00f, 9.81f, 0.818f, 0.831f},
    {32, 16, 4, 2, 2.27f, 0.00f, 1.87f, 0.236f, 0.278f},   {128, 64, 2, 1, 1.41f, 1.79f, 1.81f, 0.394f, 0.309f}};
static const Fp8Form FORMS_32[] = {
    {16, 16, 4, 4, 2.14f, 0.00f, 1.45f, 0.280f, 0.365f},   {16, 16, 8, 2, 2.06f, 0.08f, 1.57f, 0.352f, 0.354f},
    {64, 16, 4, 1, 1.43f, 1.08f, 0.96f, 0.539f, 0.063f},   {64, 32, 4, 1, 1.72f, 0.87f, 2.03f, 0.763f, 0.055f},
    {64, 64, 2, 2, 2.39f, 0.00f, 2.47f, 0.563f, 0.643f},   {128, 128, 1, 2, 2.92f, 0.00f, 5.26f, 0.628f, 1.111f},
    {64, 64, 4, 1, 1.74f, 0.81f, 2.38f, 1.051f, 0.252f},   {128, 128, 2, 1, 2.43f, 0.00f, 5.55f, 1.261f, 0.514f}};

template <typename T>
static nq_status launch_gemm(const Fp8GemmParams &p, const Fp8Launch &s)
{
    constexpr bool F32 = sizeof(T) == 4;
    const Fp8Form *forms = F32 ? FORMS_32 : FORMS_16;
    const int count = F32 ? 8 : 12;
    int best = 0;
    double least = 1e300;
    for (int i = 0; i < count; ++i) {
        const double t = form_time(forms[i], p.M, p.N, p.KB);
        if (t < least) {
            least = t;
            best = i;
        }
    }
    note_last_kernel(FP8_FAMILY, best);
    switch (best) {
    case 0: return launch_tile<T, 16, 16, 16, 16, 4, 2, 1, false>(p, s);
    case 1: return launch_tile<T, 16, 16, 16, 16, 8, F32 ? 2 : 3, 2, false>(p, s);
    case 2: return launch_tile<T, 64, 16, 32, 16, 4, 3, 2, false>(p, s);
    case 3: return launch_tile<T, 64, 32, 32, 16, 4, 3, 4, false>(p, s);
    case 4: return launch_tile<T, 64, 64, 32, 32, 2, 2, 2, false>(p, s);
    case 5: return launch_tile<T, 128, 128, 64, 64, 1, 2, 2, true>(p, s);
    default: break;
    }
    if constexpr (F32) {
        if (best == 6) return launch_tile<T, 64, 64, 32, 32, 4, 2, 4, false>(p, s);
        return launch_tile<T, 128, 128, 64, 64, 2, 2, 2, true>(p, s);
    } else {
        switch (best) {
        case 6: return launch_tile<T, 64, 64, 32, 32, 2, 3, 2, false>(p, s);
        case 7: return launch_tile<T, 128, 128, 64, 32, 1, 3, 2, true>(p, s);
        case 8: return launch_tile<T, 256, 128, 64, 64, 1, 3, 2, true>(p, s);
        case 9: return launch_tile<T, 256, 256, 128, 64, 1, 2, 2, true>(p, s);
        case 10: return launch_tile<T, 32, 16, 16, 16, 4, 3, 2, false>(p, s);
        default: return launch_tile<T, 128, 64, 64, 32, 2, 3, 2, true>(p, s);
        }
    }
}

constexpr int64_t FP8_N_STEP = 1 << 20;                    // weight rows of a launch: whole tiles and blocks of 128

}  // namespace nq

using namespace nq;

extern "C" nq_status nq_gemm_fp8(const nq_fp8 *x, const nq_fp8 *w, const float *d_bias, void *d_y, int dtype, int64_t ldy,
                                 void *stream)
{
    if (!is_dtype(dtype)) return NQ_ERR_INVALID_ARG;
    nq_status st;
    if ((st = check_fp8(x)) != NQ_OK || (st = check_fp8(w)) != NQ_OK) return st;
    if (x->block_rows != 1 || w->block_rows != 128) return NQ_ERR_UNSUPPORTED;
    if (x->cols != w->cols || w->rows > (int64_t(1) << 30)) return NQ_ERR_SHAPE;
    if (x->rows == 0 || w->rows == 0) return NQ_OK;
    if ((st = check_matrix(d_y, dtype, w->rows, ldy)) != NQ_OK) return st;
    if (!aligned_to(d_bias, 4)) return NQ_ERR_ALIGN;

    Fp8GemmParams p;
    p.ldx = x->ld;
    p.ldw = w->ld;
    p.ldy = ldy;
    p.sxr = x->scale_row_step;
    p.sxc = x->scale_col_step;
    p.swr = w->scale_row_step;
    p.swc = w->scale_col_step;
    p.K = (int)w->cols;
    p.KB = (p.K + 127) / 128;
    const int es = dtype_bytes(dtype);
    // The tiles need rows on 16 bytes and scales that a buffer descriptor reaches from a tile's first token on.
    const int64_t span = (255 * p.sxr + (int64_t)std::max(0, p.KB - 1) * p.sxc + 1) * 4;
    const bool tiled = p.KB > 0 && aligned16(x->d_q) && aligned16(w->d_q) && x->ld % 16 == 0 && w->ld % 16 == 0 && span < (int64_t(1) << 30);
    p.sx_span = tiled ? (int)span : 0;
    // A dispatch has fewer than 2^32 threads: at most 2^22 tiles of 16 x 16, of up to 512 threads, go to one; whole tiles of every form.
    Fp8Launch at{(hipStream_t)stream, nullptr, nullptr};
    void *start, *stop;                                    // (of the first and of the last launch)
    take_profile_events(&start, &stop);
    for (int64_t n = 0; n < w->rows; n += FP8_N_STEP) {
        p.N = (int)std::min(FP8_N_STEP, w->rows - n);
        p.w = w->d_q ? w->d_q + n * w->ld : nullptr;
        p.sw = w->d_scale ? w->d_scale + n / 128 * w->scale_row_step : nullptr;
        p.bias = d_bias ? d_bias + n : nullptr;
        const int64_t step = std::min<int64_t>(1 << 24, (1 << 22) / ceil_div(p.N, 16) * 16 / 256 * 256);
        for (int64_t m = 0; m < x->rows; m += step) {
            p.M = (int)std::min<int64_t>(step, x->rows - m);
            p.x = x->d_q ? x->d_q + m * x->ld : nullptr;
            p.sx = x->d_scale ? x->d_scale + m * x->scale_row_step : nullptr;
            p.y = static_cast<uint8_t *>(d_y) + (m * ldy + n) * es;
            at.start = n == 0 && m == 0 ? start : nullptr;
            at.stop = n + p.N == w->rows && m + p.M == x->rows ? stop : nullptr;
            if (dtype == NQ_DT_F32)
                st = tiled ? launch_gemm<float>(p, at) : launch_any<float>(p, at);
            else if (dtype == NQ_DT_F16)
                st = tiled ? launch_gemm<_Float16>(p, at) : launch_any<_Float16>(p, at);
            else
                st = tiled ? launch_gemm<bf16_t>(p, at) : launch_any<bf16_t>(p, at);
            if (st != NQ_OK) return st;
        }
    }
    return NQ_OK;
}
