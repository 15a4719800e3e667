// The e4m3 matrix product: tiles of BN weight rows x BM tokens through LDS.
//
// Both operands travel global -> LDS directly (buffer loads with the LDS bit) into a ring of STAGES stages, each holding G
// blocks of 128 columns of the tile's rows.  A wave-wide load writes 1024 contiguous bytes, eight rows; a row's eight 16-byte
// pieces lie exchanged, piece c at c ^ ((row / 2) & 7): two rows are once round the 64 banks, and the same piece of sixteen
// rows lies in sixteen different places.  Rows past the matrix's end, and pieces past a row's, are requested out of range and
// arrive as zeros; the bytes past a row's end inside its last piece are cleared in LDS.  The waves are G groups of
// (BN / WN) x (BM / WM); group g takes the column blocks g, g + G, ..., so that a tile has G times the waves where there are
// too few tiles to fill the card, and the groups' sums are added in order at the end.
//
// AHEAD, for the large tiles: a step does not begin with its barrier but has it as soon as all its weights are in registers, so that the
// next step's first fragments are read while the matrix cores still work; the loads of the stage to come are issued one at a time
// between the products (a burst of them holds the wave at the address unit); and four products are in flight, each one's multiply-adds
// standing behind the third product after it.  8192^3 507 -> 475 us, 1024 x 8192 x 8192 89 -> 68 (its tile then 256 x 128, in
// three stages), 512 x 8192 x 4096 24.8 -> 22.7.  Tiles of a few products to a step have more waves instead.
#pragma once
#include "nq_fp8_gemm.h"

namespace nq {

constexpr uint32_t F8_OOR = 0x7fff0000;                  // beyond every descriptor's range: reads as zeros

// Tile number -> (tile row, tile column).  Workgroups are dealt to the eight XCDs in turn, and each XCD has an L2 of its own: it
// gets a contiguous run of tiles, ordered in bands of eight tile rows so that what runs together shares both operands.
__device__ __forceinline__ void f8_tile_of(int id, int rows, int cols, int &bm, int &bn)
{
    const int total = rows * cols, each = total >> 3, more = total & 7, xcd = id & 7, at = id >> 3;
    const int t = xcd * each + min(xcd, more) + at;
    if (rows == 1) {                                     // (few tokens: no divisions)
        bm = 0;
        bn = t;
        return;
    }
    const int band = t / (8 * cols), in_band = t - band * 8 * cols, height = min(8, rows - band * 8);
    bn = in_band / height;
    bm = band * 8 + in_band - bn * height;
}

template <typename T, int BN, int BM, int WN, int WM, int G, int STAGES, int OCC, bool AHEAD>
__global__ void __launch_bounds__(64 * G * (BN / WN) * (BM / WM), OCC) k_fp8_gemm_tile(const Fp8GemmParams p)
{
    constexpr bool WIDE = sizeof(T) == 4;
    constexpr int WAVES_N = BN / WN, WAVES_M = BM / WM, GROUP = WAVES_N * WAVES_M, WAVES = G * GROUP;
    constexpr int TN = WN / 16, TM = WM / 16;
    constexpr int SX = (BM < 64 ? 64 : BM) * 4;          // bytes of a block's token scales
    constexpr int KBYTES = (BN + BM) * 128, STAGE = G * (KBYTES + SX);
    constexpr int LOADS_W = BN / 8 / GROUP, LOADS_X = BM / 8 / GROUP;    // loads of a wave and stage, of its own group's block
    static_assert(LOADS_W * GROUP * 8 == BN && LOADS_X * GROUP * 8 == BM, "the waves of a group share its loads evenly");
    static_assert(WN <= 128 && 128 % WN == 0, "a wave's weights share a scale");

    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    typedef __attribute__((address_space(3))) void *lds_ptr;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = wave / GROUP, in_group = wave - group * GROUP;
    const int wn = (in_group % WAVES_N) * WN, wm = (in_group / WAVES_N) * WM;
    const int r16 = lane & 15, g4 = lane >> 4;
    int bm, bn;
    f8_tile_of(blockIdx.x, (p.M + BM - 1) / BM, (p.N + BN - 1) / BN, bm, bn);
    const int m0 = bm * BM, n0 = bn * BN;
    const int iters = (p.KB + G - 1) / G;

    // ---- what this wave loads: rows [8 * LOADS_* * in_group, + 8 * LOADS_*) of either operand ---------------------
    auto uniform_ptr = [](const void *q) {
        const uint64_t a = reinterpret_cast<uint64_t>(q);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
        return reinterpret_cast<void *>(((uint64_t)hi << 32) | lo);
    };
    const int ldw = (int)p.ldw, ldx = (int)p.ldx;
    const __amdgpu_buffer_rsrc_t w_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        uniform_ptr(p.w + n0 * p.ldw), 0, __builtin_amdgcn_readfirstlane(min(BN, p.N - n0) * ldw), 0x00020000);
    const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        uniform_ptr(p.x + m0 * p.ldx), 0, __builtin_amdgcn_readfirstlane(min(BM, p.M - m0) * ldx), 0x00020000);
    const int first_w = in_group * LOADS_W, first_x = in_group * LOADS_X;
    // (where the loads come in pairs, those of either operand begin with an even one and share the exchange of pieces)
    constexpr bool PAIRS = LOADS_W % 2 == 0 && LOADS_X % 2 == 0;
    int piece_w[2], piece_x[2];                          // of the rows of even and of odd loads
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        piece_w[i] = 16 * ((lane & 7) ^ ((4 * ((PAIRS ? i : first_w + i) & 1) + (lane >> 4)) & 7));
        piece_x[i] = PAIRS ? piece_w[i] : 16 * ((lane & 7) ^ ((4 * ((first_x + i) & 1) + (lane >> 4)) & 7));
    }
    // the token scales of the group's block: every wave asks for 64 of them (several waves for the same ones)
    const int sx_at = (in_group % (SX / 256)) * 64 + lane;
    const bool sx_in = sx_at < BM && m0 + sx_at < p.M;
    const __amdgpu_buffer_rsrc_t sx_rsrc =
        __builtin_amdgcn_make_buffer_rsrc(uniform_ptr(p.sx + m0 * p.sxr), 0, __builtin_amdgcn_readfirstlane(p.sx_span), 0x00020000);

    // A lane's offsets stay the same from block to block, whose own offset is the scalar one: a step costs no vector instruction for
    // its addresses.  From a row's last block on the pieces past its end, and then all of them, are asked for out of range.  (The
    // range check takes the scalar offset from the range and would wrap, were that past the end: it stays at the last block.)
    constexpr int PER_STAGE = LOADS_W + LOADS_X + 1;
    uint32_t off[PER_STAGE];
#pragma unroll
    for (int l = 0; l < LOADS_W; ++l) off[l] = (8 * (first_w + l) + (lane >> 3)) * ldw + piece_w[l & 1];
#pragma unroll
    for (int l = 0; l < LOADS_X; ++l) off[LOADS_W + l] = (8 * (first_x + l) + (lane >> 3)) * ldx + piece_x[l & 1];
    off[PER_STAGE - 1] = sx_in ? (uint32_t)sx_at * (uint32_t)p.sxr * 4u : F8_OOR;
    uint8_t *const mine = lds + group * (KBYTES + SX);
    const int last_kb = p.KB - 1;
    const uint32_t sx_col = (uint32_t)p.sxc * 4u;
    int kb = group, k_at = min(group, last_kb) * 128;
    uint32_t sx_from = (uint32_t)min(group, last_kb) * sx_col;
    auto next_block = [&](bool first = false) {
        if (!first) {
            kb += G;
            if (kb <= last_kb) {
                k_at += G * 128;
                sx_from += G * sx_col;
            }
        }
        if (kb >= last_kb) {
            const int here = kb == last_kb ? p.K - last_kb * 128 : 0;
#pragma unroll
            for (int l = 0; l < PER_STAGE; ++l) {
                const int piece = l < LOADS_W ? piece_w[l & 1] : l < LOADS_W + LOADS_X ? piece_x[(l - LOADS_W) & 1] : 0;
                off[l] = piece < here ? off[l] : F8_OOR;
            }
        }
    };
    // loads [from, to) of the block into the stage at `at`
    auto issue = [&](int at, int from, int to) {
        uint8_t *dst = mine + at;
#pragma unroll
        for (int l = 0; l < PER_STAGE; ++l) {
            if (l < from || l >= to) continue;
            if (l < LOADS_W)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (lds_ptr)(dst + (first_w + l) * 1024), 16, (int)off[l], k_at, 0, 0);
            else if (l < LOADS_W + LOADS_X)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rsrc, (lds_ptr)(dst + BN * 128 + (first_x + l - LOADS_W) * 1024), 16, (int)off[l], k_at, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(sx_rsrc, (lds_ptr)(dst + KBYTES + (in_group % (SX / 256)) * 256), 4, (int)off[l], (int)sx_from, 0, 0);
        }
    };

    // (small tiles: the biases are there when the sums are)
    f8_f4 bias[TN];
    if (TN <= 2 && group == 0) fp8_bias(p, n0 + wn, lane, bias);

    // ---- the product -----------------------------------------------------------------------------------------
    f8_f4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f8_f4{0.0f, 0.0f, 0.0f, 0.0f};
    const int s8 = (r16 >> 1) & 7;
    const int at_lo = r16 * 128 + 16 * (g4 ^ s8), at_hi = r16 * 128 + 16 * ((g4 + 4) ^ s8);
    const float *sw_row = p.sw + (int64_t)((n0 + wn) >> 7) * p.swr;
    if (n0 + wn >= p.N) sw_row = p.sw;                   // (zeros times any scale: nothing of it is stored)

    // (a group without a block in the last step adds zeros times a scale of zero)
    const float *sw_at = sw_row + (int64_t)min(group, last_kb) * p.swc;
    const int64_t sw_step = G * p.swc;
    int sw_kb = group;
    auto scale_at = [&] { return G == 1 || sw_kb <= last_kb ? *sw_at : 0.0f; };
    auto next_scale = [&] {
        sw_kb += G;
        if (sw_kb <= last_kb) sw_at += sw_step;
        return scale_at();
    };
    auto frag = [&](const uint8_t *rows) {
        return fp8_frag(*reinterpret_cast<const f8_v4i *>(rows + at_lo), *reinterpret_cast<const f8_v4i *>(rows + at_hi));
    };
    // Stage `it` for everybody.  Loads complete in order and every step asks for as many (those past the end for nothing), so this many
    // outstanding means that this wave's rows have arrived.  Where the last piece of a row ends before its sixteenth byte, the wave that
    // loaded it clears what is behind.
    const int cut_it = p.K % 16 != 0 && (p.KB - 1) % G == group ? (p.KB - 1) / G : -1;
    auto arrived = [&](int it, int at, bool first = false) {
        constexpr int LEFT = (STAGES - 2) * PER_STAGE, FIRST = (STAGES - 1) * PER_STAGE;
        __builtin_amdgcn_sched_barrier(0);
        if (first)                                       // (before the loop, with every stage asked for)
            __builtin_amdgcn_s_waitcnt((FIRST & 15) | (7 << 4) | (0 << 8) | ((FIRST >> 4) << 14));
        else
            __builtin_amdgcn_s_waitcnt((LEFT & 15) | (7 << 4) | (0 << 8) | ((LEFT >> 4) << 14));
        if (it == cut_it) {
            for (int i = lane; i < 8 * (LOADS_W + LOADS_X); i += 64) {
                const int r = i < 8 * LOADS_W ? 8 * first_w + i : BN + 8 * first_x + i - 8 * LOADS_W;
                uint8_t *q = mine + at + r * 128 + 16 * (((p.K & 127) >> 4) ^ ((r >> 1) & 7));
                for (int b = p.K & 15; b < 16; ++b) q[b] = 0;
            }
            __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();                    // (alone: __syncthreads() would wait for the stages on their way as well)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // stages by where they begin
    auto after = [&](int at) { return at == (STAGES - 1) * STAGE ? 0 : at + STAGE; };
    auto before = [&](int at) { return at == 0 ? (STAGES - 1) * STAGE : at - STAGE; };

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        next_block(s == 0);
        issue(s * STAGE, 0, PER_STAGE);
    }
    float sw = scale_at();
    if constexpr (!AHEAD) {
        for (int it = 0, at = 0; it < iters; ++it, at = after(at)) {
            arrived(it, at);
            const float sw_next = next_scale();          // (before the stage's loads: complete when they are waited for)
            next_block();
            issue(before(at), 0, PER_STAGE);
            const uint8_t *cur = mine + at;
            const float *sxp = reinterpret_cast<const float *>(cur + KBYTES) + wm + r16;
            Fp8Operand<WIDE> x[TM];
            float s[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                x[i].set(frag(cur + (BN + wm + 16 * i) * 128));
                s[i] = sxp[i * 16] * sw;
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                Fp8Operand<WIDE> w;
                w.set(frag(cur + (wn + 16 * j) * 128));
#pragma unroll
                for (int i = 0; i < TM; ++i) fp8_add(acc[i][j], fp8_mfma(w, x[i]), s[i]);
            }
            sw = sw_next;
        }
    } else {
        // Product k of a step is weight fragment k / TM with token fragment k % TM.  The weights go round a ring, RING - 1 fragments ahead;
        // from fragment TURN on, when all of a stage's are in registers, they are the next stage's, and its own place is filled again.  A
        // fragment of tokens is read for the next step as soon as its last product is under way, and a product's multiply-adds
        // stand DEPTH products after it, those of a step's last ones in the next step.
        constexpr int COUNT = TN * TM, DEPTH = 3, RING = TN % 4 == 0 ? 4 : 2, TURN = TN - RING + 1;
        constexpr int SPREAD = COUNT / 4 < COUNT - TURN * TM ? COUNT / 4 : COUNT - TURN * TM;
        static_assert(TN % RING == 0 && COUNT % (DEPTH + 1) == 0, "fragments and products have the same places in every step");
        static_assert(COUNT - TM > DEPTH, "a step's scales are taken before the next one's are read");
        f8_v8i wf[RING], xf[TM];
        Fp8Operand<WIDE> w, x[TM];
        f8_f4 prod[DEPTH + 1];
        float s[TM], sx[TM];
        auto tokens = [&](int i, int at) {
            xf[i] = frag(mine + at + (BN + wm + 16 * i) * 128);
            sx[i] = reinterpret_cast<const float *>(mine + at + KBYTES)[wm + r16 + 16 * i];
        };
        auto weights = [&](int j, int at) { wf[j % RING] = frag(mine + at + (wn + 16 * j) * 128); };
        auto add = [&](int k) {
            fp8_add(acc[k % TM][k / TM], prod[k % (DEPTH + 1)], s[k % TM]);
            asm volatile("" : "+v"(acc[k % TM][k / TM]));       // (here: not sunk to the loop's end, with its product kept until then)
        };
        float sw_then = next_scale();
        next_block();
        issue((STAGES - 1) * STAGE, 0, PER_STAGE);
        arrived(0, 0, true);
#pragma unroll
        for (int j = 0; j < RING - 1; ++j) weights(j, 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) tokens(i, 0);
#pragma unroll
        for (int i = 0; i <= DEPTH; ++i) prod[i] = f8_f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < TM; ++i) s[i] = 0.0f;
        for (int it = 0, at = 0; it < iters; ++it, at = after(at)) {
            float sw_next = 0.0f;
#pragma unroll
            for (int k = 0; k < COUNT; ++k) {
                const int j = k / TM, i = k % TM;
                if (i == 0) {
                    if (j == TURN) {                     // all weights of this stage are in registers
                        arrived(it + 1, after(at));
                        sw_next = next_scale();
                        next_block();
                    }
                    w.set(wf[j % RING]);
                    if (j + RING - 1 < TN) weights(j + RING - 1, at);
                    else weights(j + RING - 1 - TN, after(at));
                }
                if (j == 0) x[i].set(xf[i]);
                prod[k % (DEPTH + 1)] = fp8_mfma(w, x[i]);
                if (j == TN - 1) tokens(i, after(at));
                if (k >= TURN * TM && k < TURN * TM + SPREAD)
                    issue(at, (k - TURN * TM) * PER_STAGE / SPREAD, (k - TURN * TM + 1) * PER_STAGE / SPREAD);
                if (k == DEPTH) {
#pragma unroll
                    for (int m = 0; m < TM; ++m) s[m] = sx[m] * sw;
                }
                add((k + COUNT - DEPTH) % COUNT);
                __builtin_amdgcn_sched_barrier(0);
            }
            sw = sw_then;
            sw_then = sw_next;
        }
#pragma unroll
        for (int k = COUNT - DEPTH; k < COUNT; ++k) add(k);
    }

    // every load has to have landed before its memory is used for something else
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));
    // ---- the groups' sums, one after the other -------------------------------------------------------------------
    __syncthreads();
    constexpr int SUMS = (G - 1) * GROUP * TM * TN * 1024;
    if constexpr (G > 1) {
        f8_f4 *sum = reinterpret_cast<f8_f4 *>(lds);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                if (group > 0) sum[(((group - 1) * GROUP + in_group) * TM * TN + i * TN + j) * 64 + lane] = acc[i][j];
        __syncthreads();
        if (group > 0) return;
        for (int g = 1; g < G; ++g)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] += sum[(((g - 1) * GROUP + in_group) * TM * TN + i * TN + j) * 64 + lane];
    }
    if (TN > 2) fp8_bias(p, n0 + wn, lane, bias);
    fp8_store_tile<T, TN, TM>(p, m0 + wm, n0 + wn, acc, bias, lds + SUMS + in_group * (TM * TN * 256 * (int)sizeof(T)), lane);
}

template <typename T, int BN, int BM, int WN, int WM, int G, int STAGES, int OCC, bool AHEAD>
static nq_status launch_tile(const Fp8GemmParams &p, const Fp8Launch &s)
{
    constexpr int GROUP = (BN / WN) * (BM / WM);
    constexpr int ring = STAGES * G * ((BN + BM) * 128 + (BM < 64 ? 64 : BM) * 4);
    constexpr int sums = (G - 1) * GROUP * (WN / 16) * (WM / 16) * 1024;
    constexpr int last = sums + BN * BM * (int)sizeof(T);
    constexpr int lds = ring > last ? ring : last;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    auto k = k_fp8_gemm_tile<T, BN, BM, WN, WM, G, STAGES, OCC, AHEAD>;
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> granted{0};
        const nq_status st = grant_lds(k, lds, granted);
        if (st != NQ_OK) return st;
    }
    return launch_fp8(s, k, ceil_div(p.M, BM) * ceil_div(p.N, BN), 64 * G * GROUP, lds, p);
}

}  // namespace nq
