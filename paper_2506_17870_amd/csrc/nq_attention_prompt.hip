// nq_attention_prompt: attention over whole prompts, packed sequences, causal or not, grouped heads.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = 2^(x_ij - m_i),  x_ij = scale log2(e) (q_i . k_j),  m_i the largest x so far
//
// Bound by the matrix core, by the exponentials next to it, and for long prompts by the card's power: 8192 causal rows of 32 heads of 128 bf16
// take 533 us (1.03 PFLOP/s, 518 to 546 us by the card's clock; the library's matrix product reaches 1.22), at 1.8 GHz with the matrix core busy 55 % of the
// time.  A workgroup takes
// 128 rows of a head, a wave 32 of them, and goes over the keys 64 (32) at a time (short calls: enum Share); two workgroups to a compute unit do one's exponentials
// beside the other's products.  Both products are transposed: S^T = K Q^T, O^T = V^T P^T.  A lane then holds scores of
// one row only, its maximum and sum need one exchange with another lane, and because the order in which a product sums its keys is
// free, the scores' places after the first product are the probabilities' places in the second one's operand: they never leave
// their registers.  The probabilities are rounded to the operands' type for it, each by half a step at most, as the matrix core wants them; over
// bf16 inputs the result is off by 2.0e-3 (2-norm), of which rounding the result itself is 1.6e-3.  K and V tiles go through LDS, V's fragments
// by the transposing read.
// Measured and not kept: 64 rows to a wave with one wave to a SIMD (721 us); the products of the next and the last 32 keys scheduled between the
// exponentials of one wave (558 us, packed prompts 147 for 140: fewer instructions, but more of a prologue, and the clock falls with the power).
#include "nq_attention.h"

namespace nq {

typedef __bf16 at_b8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_h2 __attribute__((ext_vector_type(2)));
typedef float at_f16 __attribute__((ext_vector_type(16)));
typedef short at_s4 __attribute__((ext_vector_type(4)));
typedef short at_s2 __attribute__((ext_vector_type(2)));

constexpr float PR_LOG2E = 1.44269504088896340736f;
// A row's maximum is moved only when a score passes it by this much (in powers of two): the probabilities are relative to it, so
// any reference will do that keeps them within their type.
constexpr float PR_SLACK = 8.0f;

struct PromptParams {
    const void *q, *k, *v;
    void *o;
    const int32_t *q_begin, *k_begin;
    int64_t ldq, ldk, ldv, ldo;
    int32_t sequences, q_rows, k_rows, Hq, Hkv, group, D, causal, tiles;   // tiles: of rows, at most
    Divider by_heads;
    float scale;                                // times log2(e), its magnitude
    uint32_t flip;                              // sign bits for q where the scale is negative
    int32_t first_half;                         // tiles of which one is on each compute unit before any has two
    int32_t zero;                               // a scale of 0
    float *partial;                             // sums of o [pieces][q_rows][q_heads][D], then m and l [pieces][q_rows][q_heads][2]
    int32_t pieces;                             // workgroups that share the keys of a tile of rows; 1: they write the rows themselves
};

template <typename T>
__device__ __forceinline__ at_f16 mma32(uint4 a, uint4 b, at_f16 c)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f8_h8, a), __builtin_bit_cast(f8_h8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(at_b8, a), __builtin_bit_cast(at_b8, b), c, 0, 0, 0);
}
template <typename T>
__device__ __forceinline__ uint32_t pair16(float a, float b)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_bit_cast(uint32_t, at_h2{(_Float16)a, (_Float16)b});
    else
        return pack_bf16(a, b);
}
template <typename T>
__device__ __forceinline__ float value16(uint16_t v)
{
    if constexpr (__is_same(T, _Float16))
        return (float)__builtin_bit_cast(_Float16, v);
    else
        return __builtin_bit_cast(float, (uint32_t)v << 16);
}
template <typename T>
__device__ __forceinline__ float sum_pair(uint32_t p, float sum)
{
    if constexpr (__is_same(T, _Float16))
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(at_h2, p), at_h2{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
    else
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(at_s2, p), __builtin_bit_cast(at_s2, 0x3f803f80u), sum, false);
}
__device__ __forceinline__ float across32(float v, bool sum)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t x = r[0], y = r[1];                                   // (a bit cast of a vector's element takes its first)
    const float a = __builtin_bit_cast(float, x), b = __builtin_bit_cast(float, y);
    return sum ? a + b : fmaxf(a, b);
}
__device__ __forceinline__ uint2 read_transposed(const uint16_t *at)
{
    typedef __attribute__((address_space(3))) at_s4 lds_s4;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)at));
}

// LDS rows of PITCH elements in pieces of 16 bytes, exchanged so that neither the rows that a wave reads at once nor the four rows of a
// transposing read meet in a bank.
template <int PITCH>
__device__ __forceinline__ int k_piece(int row, int piece) { return piece ^ (PITCH == 64 ? (row ^ (row >> 3 & 3)) & 7 : row & 15); }
template <int PITCH>
__device__ __forceinline__ int v_piece(int row, int piece) { return piece ^ (PITCH == 64 ? (row & 2) << 1 : ((row & 3) << 2) | ((row >> 2) & 3)); }

constexpr int pitch_of(int DP) { return DP <= 64 ? 64 : DP <= 128 ? 128 : 256; }
// How a workgroup's waves share its work.  ROWS: four waves of 32 rows each; KEYS: of the same 32 rows, the keys dealt to them; ALONE: one wave of
// 32 rows.  Keys of a step: as many as the registers hold beside the outputs.
enum Share { SHARE_ROWS, SHARE_KEYS, SHARE_ALONE };
constexpr int stages_of(int DP, Share share) { return share == SHARE_ALONE || (share == SHARE_KEYS && DP > 64) ? 1 : 2; }
constexpr int keys_of(int DP, Share share) { return share == SHARE_ALONE ? 32 : share == SHARE_KEYS ? 128 : DP <= 128 ? 64 : 32; }
constexpr int waves_of(Share share) { return share == SHARE_ALONE ? 1 : 4; }

// Which rows a workgroup takes: number w in the order of the keys that they see, the most first (in steps of PR_LEVEL keys), so that what
// is left for the end is short; where all fit on the card at once, two to a compute unit, the second ones the fewest first (2048 rows of 32 heads 50.4
// us and 48.2 so, 1500 37.0 and 35.4).  For up to PR_PLANNED sequences, a lane each of 64; every wave makes the same sums.
constexpr int PR_LEVEL = 512, PR_PLANNED = 256;
struct Rows {
    int sequence, tile;                          // -1: none
};
template <int ROWS>
__device__ __forceinline__ Rows rows_of(const PromptParams &p, int w)
{
    const int lane = threadIdx.x & 63;
    if (p.sequences > PR_PLANNED) {
        // in the order of the sequences from the last on: tile t belongs to the last sequence s with begin / ROWS + s <= t (begins in front of the rows: 0)
        const int t = p.tiles - 1 - w;
        auto first_of = [&](int s) { return max(p.q_begin[s], 0) / ROWS + s; };      // (under 2^31: sequences are under 2^30)
        int lo = -1, hi = p.sequences;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_of(mid) <= t) lo = mid; else hi = mid;
        }
        return lo < 0 ? Rows{-1, 0} : Rows{lo, t - first_of(lo)};
    }
    if (p.sequences == 1) {
        const int q0 = min(max(p.q_begin[0], 0), p.q_rows), n = (min(max(p.q_begin[1], q0), p.q_rows) - q0 + ROWS - 1) / ROWS;
        if (w < n && w >= p.first_half && n <= 2 * p.first_half) w = n - 1 - (w - p.first_half);
        return Rows{w < n ? 0 : -1, n - 1 - w};
    }
    constexpr int CH = PR_PLANNED / 64;
    int tiles[CH], keys[CH], ahead[CH], most = 0, total = 0, all;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = 64 * c + lane;
        tiles[c] = keys[c] = ahead[c] = 0;
        if (i < p.sequences) {
            const int q0 = min(max(p.q_begin[i], 0), p.q_rows), Lq = min(max(p.q_begin[i + 1], q0), p.q_rows) - q0;
            const int k0 = min(max(p.k_begin[i], 0), p.k_rows);
            keys[c] = min(max(p.k_begin[i + 1], k0), p.k_rows) - k0;
            tiles[c] = (Lq + ROWS - 1) / ROWS;
            ahead[c] = keys[c] - Lq;
        }
        total += tiles[c];
        most = max(most, keys[c]);
    }
    (void)before(total, &all);
    if (w >= all) return Rows{-1, 0};
    if (w >= p.first_half && all <= 2 * p.first_half) w = all - 1 - (w - p.first_half);
    // tiles of a sequence that see more than (x - 1) * PR_LEVEL keys, the last ones of it
    auto count = [&](int c, int x) {
        if (x == 0) return tiles[c];
        const int y = (x - 1) * PR_LEVEL + 1;
        if (keys[c] < y) return 0;
        return p.causal ? min(tiles[c], tiles[c] - (max(y - ahead[c], 1) + ROWS - 1) / ROWS + 1) : tiles[c];
    };
    auto sum = [&](int x) {
        int n = 0, s;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (64 * c < p.sequences) n += count(c, x);
        (void)before(n, &s);
        return s;
    };
#pragma unroll
    for (int k = 1; k < 64; k *= 2) most = max(most, __shfl_xor(most, k));
    int x = 0, hi = __builtin_amdgcn_readfirstlane(most) / PR_LEVEL + 2, more = 0;    // sum(x) > w >= sum(hi) == more
    while (hi - x > 1) {
        const int mid = (x + hi) >> 1, s = sum(mid);
        if (s > w) {
            x = mid;
        } else {
            hi = mid;
            more = s;
        }
    }
    int at = w - more;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int upper = 64 * c < p.sequences ? count(c, x + 1) : 0, here = 64 * c < p.sequences ? count(c, x) - upper : 0, first = before(here, &all);
        const uint64_t mask = __ballot(at >= first && at < first + here);
        if (mask) {
            const int from = __builtin_ctzll(mask);
            return Rows{64 * c + from, __builtin_amdgcn_readlane(tiles[c] - upper - here + at - first, from)};
        }
        at -= all;
    }
    return Rows{-1, 0};
}

// The same for SHARE_ALONE, whose sequences have one tile mostly: nothing to look for there.  Behind the first 32 rows of each come as many tiles as
// multiples of 32 lie in the call's rows: that of x belongs to the sequence with rows on both sides of x, which has one for each such tile.
__device__ __forceinline__ Rows rows_alone(const PromptParams &p, int w)
{
    const int t = p.q_rows / 32 - w;                                     // the multiple 32 t, the last first
    if (t <= 0) return Rows{-t, 0};
    int lo = -1, hi = p.sequences;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.q_begin[mid] < 32 * t) lo = mid; else hi = mid;
    }
    return lo < 0 ? Rows{-1, 0} : Rows{lo, t - max(p.q_begin[lo], 0) / 32};
}

// DIRECT: K and V travel global -> LDS by direct loads a step ahead, which want rows on 16 bytes; else through registers, when they are used.
// DEALT: the keys that a tile of rows sees are dealt to p.pieces workgroups, which leave their sums to k_prompt_join.
template <typename T, int DP, Share SHARE, bool DIRECT, bool DEALT>
__global__ void __launch_bounds__(waves_of(SHARE) * 64, DP > 128 ? 1 : SHARE == SHARE_KEYS || DP > 64 ? 2 : 3) k_attention_prompt(const PromptParams p)
{
    constexpr bool SPLIT = SHARE == SHARE_KEYS;
    constexpr int PITCH = pitch_of(DP), KEYS = keys_of(DP, SHARE), STAGES = stages_of(DP, SHARE), U = SPLIT ? 1 : KEYS / 32, KJ = DP / 16, DT = DP / 32;
    constexpr int WAVES = waves_of(SHARE), THREADS = WAVES * 64, ROWS = SHARE == SHARE_ROWS ? 128 : 32, TILE = KEYS * PITCH;
    constexpr int PIECES = DIRECT ? PITCH / 8 : DP / 8, CH = KEYS * PIECES / THREADS;  // pieces of 16 bytes of a row; of a thread and tile
    constexpr bool THROUGH = SHARE == SHARE_ROWS && DP <= 128;           // Q travels through LDS, too, and O where it leaves as rows
    constexpr int SUMS = SPLIT ? 1024 + 2 * 64 * (DP / 2 + 1) * 4 : 0;    // bytes for the waves' sums
    constexpr bool F16 = __is_same(T, _Float16);
    constexpr uint32_t EXP = F16 ? 0x7c00 : 0x7f80;                      // the exponent of infinities and NaN
    constexpr int NOWHERE = 0x7fffffff, RANGE = 0x7ffffff0;
    typedef __attribute__((address_space(3))) void *lds_ptr;
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[];     // two stages of K and V
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5;

    // Neighbouring workgroups take the heads in turn, those of one key head on one of the eight dies, whose cache then holds its keys.
    const uint32_t number = divide(blockIdx.x, p.by_heads);
    uint32_t h = blockIdx.x - number * p.by_heads.d;
    if (p.Hq % 8 == 0) h = (h & 7) * (p.Hq >> 3) + (h >> 3);
    const Rows mine = SHARE == SHARE_ALONE ? rows_alone(p, (int)number) : rows_of<ROWS>(p, (int)number);
    if (mine.sequence < 0) return;
    const int lo = mine.sequence, first = mine.tile;
    const int q0 = min(max(p.q_begin[lo], 0), p.q_rows), q1 = min(max(p.q_begin[lo + 1], q0), p.q_rows), Lq = q1 - q0;
    const int k0 = min(max(p.k_begin[lo], 0), p.k_rows), k1 = min(max(p.k_begin[lo + 1], k0), p.k_rows), Lk = k1 - k0;
    if (first < 0 || (int64_t)first * ROWS >= Lq) return;
    const int row0 = first * ROWS, off = p.causal ? Lk - Lq : Lk;        // row i sees the keys j <= i + off (without causal: all)
    const int end = min(Lk, max(0, min(row0 + ROWS, Lq) + off));         // keys that any row sees
    const int hk = (int)h / p.group;
    int from = 0, to = end;                                              // this workgroup's keys
    if constexpr (DEALT) {
        const int size = ((end + p.pieces - 1) / p.pieces + KEYS - 1) / KEYS * KEYS;
        from = min((int)blockIdx.y * size, end);
        to = min(from + size, end);
    }

    const T *k_base = static_cast<const T *>(p.k) + (int64_t)k0 * p.ldk + (int64_t)hk * p.D;
    const T *v_base = static_cast<const T *>(p.v) + (int64_t)k0 * p.ldv + (int64_t)hk * p.D;
    // ---- a tile's way into LDS
    int k_off[DIRECT ? CH : 1], v_off[DIRECT ? CH : 1];
    if constexpr (DIRECT) {
        // a wave's 64 pieces land beside each other: which piece of the row a lane asks for makes the exchange
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int id = (wave * CH + i) * 64 + lane, row = id / PIECES, piece = id % PIECES;
            const int kd = k_piece<PITCH>(row, piece) * 8, vd = v_piece<PITCH>(row, piece) * 8;
            k_off[i] = kd < p.D ? (int)(row * p.ldk + kd) * 2 : NOWHERE;
            v_off[i] = vd < p.D ? (int)(row * p.ldv + vd) * 2 : NOWHERE;
        }
    }
    auto fetch = [&](int j0, uint16_t *kt) __attribute__((always_inline)) {
        if constexpr (DIRECT) {
            uint16_t *vt = kt + TILE;
            const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(k_base + (int64_t)j0 * p.ldk), 0, RANGE, 0x00020000);
            const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(v_base + (int64_t)j0 * p.ldv), 0, RANGE, 0x00020000);
            const int rows = end - j0;                                   // (rows that are not there: zeros)
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int row = ((wave * CH + i) * 64 + lane) / PIECES;
                const int at = rows >= KEYS || row < rows ? k_off[i] : NOWHERE;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_ptr)(kt + (wave * CH + i) * 512), 16, at, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int row = ((wave * CH + i) * 64 + lane) / PIECES;
                const int at = rows >= KEYS || row < rows ? v_off[i] : NOWHERE;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_ptr)(vt + (wave * CH + i) * 512), 16, at, 0, 0, 0);
            }
        }
    };
    // A key that only some rows see has probability 0 in the others, and 0 times an infinite or NaN value is no 0.  So such values become zeros
    // in the tiles of those keys, and are added at the end to the rows that see them.  Where all rows see all keys there are no such tiles, also where the
    // last one has places behind the keys (zeros): a value that every row sees stays.
    int partial = row0 + 1 + off;                                        // keys that all rows see, where some rows see more
    if (partial >= to) partial = NOWHERE;
    asm("" : "+s"(partial));                                             // (one number, compared once a step: else the compiler compares twice, 3 % at 256 columns)
    uint32_t *const odd_of = reinterpret_cast<uint32_t *>(lds + (STAGES * 2 * TILE > SUMS / 2 ? STAGES * 2 * TILE : SUMS / 2));    // for each wave: whether it found such values
    if (lane == 0) odd_of[wave] = 0;
    // (what is infinite or NaN of a pair of values, zeros for the rest)
    auto not_finite = [&](uint32_t x) __attribute__((always_inline)) { return ((x & EXP) == EXP ? x & 0xffffu : 0u) | ((x >> 16 & EXP) == EXP ? x & 0xffff0000u : 0u); };
    auto tame = [&](uint4 &w) __attribute__((always_inline)) {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) found |= (x[i] & (EXP << 16 | EXP)) + ((EXP & -EXP) << 16 | (EXP & -EXP));     // (a carry out of an exponent of ones)
        if (!(found & 0x80008000u)) return false;
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = ((x[i] & EXP) == EXP ? 0u : x[i] & 0xffffu) | ((x[i] >> 16 & EXP) == EXP ? 0u : x[i] & 0xffff0000u);
        w = make_uint4(y[0], y[1], y[2], y[3]);
        odd_of[wave] = 1;
        return true;
    };
    // the tile of the keys from j0 on for everybody
    auto arrived = [&](int stage, int j0) __attribute__((always_inline)) {
        uint16_t *kt = lds + stage * 2 * TILE, *vt = kt + TILE;
        if constexpr (DIRECT) {
            __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));         // all loads, all LDS accesses
            if (j0 + KEYS > partial) {
#pragma unroll
                for (int i = 0; i < CH; ++i) {                           // (what this lane has asked for)
                    uint4 *at = reinterpret_cast<uint4 *>(vt + (wave * CH + i) * 512 + lane * 8), w = *at;
                    if (tame(w)) *at = w;
                }
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int id = i * THREADS + threadIdx.x, row = id / PIECES, piece = id % PIECES, d = piece * 8;
                uint4 k = make_uint4(0, 0, 0, 0), v = make_uint4(0, 0, 0, 0);
                if (j0 + row < end && d < p.D) {
                    __builtin_memcpy(&k, k_base + (int64_t)(j0 + row) * p.ldk + d, 16);
                    __builtin_memcpy(&v, v_base + (int64_t)(j0 + row) * p.ldv + d, 16);
                }
                if (j0 + KEYS > partial) (void)tame(v);
                *reinterpret_cast<uint4 *>(kt + row * PITCH + k_piece<PITCH>(row, piece) * 8) = k;
                *reinterpret_cast<uint4 *>(vt + row * PITCH + v_piece<PITCH>(row, piece) * 8) = v;
            }
        }
        __syncthreads();
    };

    if (from < to) fetch(from, lds);
    // this wave's rows, this lane's row
    const int first_row = row0 + (SPLIT ? 0 : wave * 32), row = first_row + r;
    uint4 q[KJ];
    const T *q_row = static_cast<const T *>(p.q) + (int64_t)(q0 + row) * p.ldq + (int64_t)h * p.D;
    uint16_t *const own = lds + 2 * TILE + wave * 32 * PITCH;            // of the second stage, free before the first step and after the last
    if constexpr (THROUGH && DIRECT) {
        // a wave's rows by whole lines, as those of K
        const T *from = static_cast<const T *>(p.q) + (int64_t)(q0 + first_row) * p.ldq + (int64_t)h * p.D;
        const __amdgpu_buffer_rsrc_t qr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(from), 0, RANGE, 0x00020000);
        constexpr int PER = PITCH / 8;
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) {
            const int at = (i * 64 + lane) / PER, d = k_piece<PITCH>(at, (i * 64 + lane) % PER) * 8;
            const int q_off = first_row + at < Lq && d < p.D ? (int)(at * p.ldq + d) * 2 : NOWHERE;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(qr, (lds_ptr)(own + i * 512), 16, q_off, 0, 0, 0);
        }
        __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));             // (this wave's alone: nobody else reads them)
#pragma unroll
        for (int j = 0; j < KJ; ++j) q[j] = *reinterpret_cast<const uint4 *>(own + r * PITCH + k_piece<PITCH>(r, 2 * j + half) * 8);
    } else {
#pragma unroll
        for (int j = 0; j < KJ; ++j) {
            const int d = 16 * j + 8 * half;
            q[j] = make_uint4(0, 0, 0, 0);
            if (row < Lq && d < p.D) __builtin_memcpy(&q[j], q_row + d, 16);
        }
    }
    if (p.zero) {                                                        // (of queries times 0 those that are not finite are left; their scores are not either)
#pragma unroll
        for (int j = 0; j < KJ; ++j) q[j] = make_uint4(not_finite(q[j].x), not_finite(q[j].y), not_finite(q[j].z), not_finite(q[j].w));
    }
    if (p.flip) {
#pragma unroll
        for (int j = 0; j < KJ; ++j) q[j] = make_uint4(q[j].x ^ p.flip, q[j].y ^ p.flip, q[j].z ^ p.flip, q[j].w ^ p.flip);
    }

    at_f16 o[DT];
    float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;

    // keys that some row of the wave sees, that all of them see; the last that this lane's row sees
    const int wave_end = first_row < Lq ? min(to, max(0, min(first_row + 32, Lq) + off)) : 0, seen_by_all = min(Lk, first_row + 1 + off);
    const int row_last = min(Lk - 1, row + off);
    // V^T of the columns 32 d .., keys 16 e + 4 half + (0 .. 3) and eight further on, as the scores lie
    auto v_fragment = [&](const uint16_t *vt, int d, int e) __attribute__((always_inline)) {
        const int at = 16 * e + 4 * half + (lane & 15) / 4, col = 32 * d + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        const uint2 x = read_transposed(vt + at * PITCH + v_piece<PITCH>(at, col >> 3) * 8 + (col & 7));
        const uint2 y = read_transposed(vt + (at + 8) * PITCH + v_piece<PITCH>(at + 8, col >> 3) * 8 + (col & 7));
        return make_uint4(x.x, x.y, y.x, y.y);
    };
    // One step: the keys from j0 on, whose tiles are kt and vt.  The two stages are named apart so that the compiler knows that what is on its
    // way into one does not hold up reading the other.
    auto step = [&](uint16_t *__restrict kt, uint16_t *__restrict vt, uint16_t *__restrict next, int j0) __attribute__((always_inline)) {
        if (STAGES == 2 && j0 + KEYS < to) fetch(j0 + KEYS, next);
        if constexpr (SPLIT) {
            j0 += wave * 32;
            kt += wave * 32 * PITCH;
            vt += wave * 32 * PITCH;
        }
        if (j0 >= wave_end) return;
        // ---- scores: lane (r, half) has row r, keys 32 u + 8 (i / 4) + 4 half + i % 4
        at_f16 s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                const int at = 32 * u + r;
                s[u] = mma32<T>(*reinterpret_cast<const uint4 *>(kt + at * PITCH + k_piece<PITCH>(at, 2 * j + half) * 8), q[j], s[u]);
            }
        }
        // (fragments are read AHEAD products before they are used)
        constexpr int AHEAD = 4;
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int i = 0; i < U * KJ - AHEAD; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
        if (j0 + 32 * U > seen_by_all) {
            const int last = row_last - j0 - 4 * half;                   // from this lane's first key on
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * u + 8 * (i / 4) + i % 4 > last) s[u][i] = -__builtin_inff();
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
        top = across32(top, false) * p.scale;
        if (__any(top > m + PR_SLACK)) {
            const float n = fmaxf(m, top), w = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - n);
            m = n;
            l *= w;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= w;
        }
        // (f16 probabilities are 2^7 times as large, 2^15 at most, so that small ones keep their bits)
        const float base = m == -__builtin_inff() ? 0.0f : m - (F16 ? 7.0f : 0.0f);
        uint4 pr[2 * U];
#pragma unroll
        for (int e = 0; e < 2 * U; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = s[e / 2][8 * (e & 1) + 2 * i], y = s[e / 2][8 * (e & 1) + 2 * i + 1];
                w[i] = pair16<T>(__builtin_amdgcn_exp2f(fmaf(x, p.scale, -base)), __builtin_amdgcn_exp2f(fmaf(y, p.scale, -base)));
                l = sum_pair<T>(w[i], l);                                // (what the second product takes, so that the weights add up to 1)
            }
            pr[e] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        // ---- V^T P^T
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 2 * U; ++e) o[d] = mma32<T>(v_fragment(vt, d, e), pr[e], o[d]);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
#pragma unroll
        for (int i = 0; i < DT * 2 * U - AHEAD; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
    };
    for (int j0 = from, stage = 0; j0 < to; j0 += KEYS, stage ^= STAGES - 1) {
        arrived(stage, j0);                                              // (and nobody reads the other stage any more)
        step(lds + stage * 2 * TILE, lds + stage * 2 * TILE + TILE, lds + (stage ^ 1) * 2 * TILE, j0);
        if (STAGES == 1 && j0 + KEYS < to) {
            __builtin_amdgcn_s_waitcnt(0xc07f);                          // (what is read is in registers before anything is on its way into its place)
            __syncthreads();
            fetch(j0 + KEYS, lds);
        }
    }
    const bool odd = partial != NOWHERE && (odd_of[0] | odd_of[WAVES / 4] | odd_of[WAVES / 2] | odd_of[WAVES - 1]);

    if constexpr (SPLIT) {
        // ---- the four waves' sums, by way of LDS: a lane's are of the same row and columns in all of them
        float *const tops = reinterpret_cast<float *>(lds), *const sums = tops + 256;
        __syncthreads();
        tops[threadIdx.x] = m;
        __syncthreads();
        const float top = fmaxf(fmaxf(tops[lane], tops[64 + lane]), fmaxf(tops[128 + lane], tops[192 + lane]));
        const float w = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        l *= w;
        m = top;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= w;
        constexpr int PER = DT * 16 + 1;
#pragma unroll
        for (int n = 2; n >= 1; n /= 2) {
            float *to = sums + (wave & (n - 1)) * 64 * PER + lane;
            if (wave >= n && wave < 2 * n) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) to[(d * 16 + i) * 64] = o[d][i];
                to[DT * 16 * 64] = l;
            }
            __syncthreads();
            if (wave < n) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] += to[(d * 16 + i) * 64];
                l += to[DT * 16 * 64];
            }
            __syncthreads();
        }
        if (wave) return;
    }

    if (odd) {
        for (int j = max(max(partial, 0) / KEYS * KEYS, from); j < to; ++j) {
            const uint16_t *values = reinterpret_cast<const uint16_t *>(v_base + (int64_t)j * p.ldv);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    const int col = 32 * d + 8 * (i / 4) + 4 * half + i % 4;
                    const uint16_t v = col < p.D ? values[col] : 0;
                    if ((v & EXP) == EXP && j <= row_last) o[d][i] += value16<T>(v);
                }
        }
    }

    // ---- lane: row r, columns 32 d + 8 (i / 4) + 4 half + i % 4
    const bool any = row_last >= 0;
    if constexpr (DEALT) {
        l = across32(l, true);
        if (row >= Lq) return;
        const int64_t at = ((int64_t)blockIdx.y * p.q_rows + q0 + row) * p.Hq + h;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int col = 32 * d + 2 * i + 4 * half;
                const float y[4] = {o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
                if (col < p.D) __builtin_memcpy(__builtin_assume_aligned(p.partial + at * p.D + col, 16), y, 16);
            }
        if (half == 0)                                                   // (a sum of -1: the row sees no key)
            reinterpret_cast<f8_f2 *>(p.partial + (int64_t)p.pieces * p.q_rows * p.Hq * p.D)[at] = f8_f2{m, any ? l : -1.0f};
        return;
    }
    // (a row whose every score is -inf has a sum of 0 and comes out as NaN, as its definition does; a row without keys as 0)
    const float w = 1.0f / across32(l, true);
    T *const out_row = static_cast<T *>(p.o) + (int64_t)(q0 + first_row) * p.ldo + (int64_t)h * p.D;     // the wave's first row
    if constexpr (THROUGH) {
        // whole rows leave, 16 bytes a lane (the second stage of the two is free where the last step was of the first, else the first)
        uint16_t *const out = lds + (end > 0 && ((end - 1) / KEYS) % 2 ? 0 : 2 * TILE) + wave * 32 * PITCH;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int col = 32 * d + 2 * i + 4 * half;
                const uint2 y = any ? make_uint2(pair16<T>(o[d][i] * w, o[d][i + 1] * w), pair16<T>(o[d][i + 2] * w, o[d][i + 3] * w)) : make_uint2(0, 0);
                *reinterpret_cast<uint2 *>(out + r * PITCH + k_piece<PITCH>(r, col >> 3) * 8 + (col & 4)) = y;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();                                 // (LDS serves a wave's requests in order)
        constexpr int PER = PITCH / 8;
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) {
            const int at = (i * 64 + lane) / PER, d = (i * 64 + lane) % PER * 8;
            const uint4 y = *reinterpret_cast<const uint4 *>(out + at * PITCH + k_piece<PITCH>(at, d >> 3) * 8);
            if (first_row + at < Lq && d < p.D) __builtin_memcpy(out_row + at * p.ldo + d, &y, 16);
        }
    } else {
        if (row >= Lq) return;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int col = 32 * d + 2 * i + 4 * half;
                const uint2 y = any ? make_uint2(pair16<T>(o[d][i] * w, o[d][i + 1] * w), pair16<T>(o[d][i + 2] * w, o[d][i + 3] * w)) : make_uint2(0, 0);
                if (col < p.D) __builtin_memcpy(out_row + r * p.ldo + col, &y, 8);
            }
    }
}

// Joins the pieces of a row and head: a thread for four columns.  Rows in front of the first sequence and behind the last have none.
template <typename T>
__global__ void __launch_bounds__(256) k_prompt_join(const PromptParams p, const Divider by_quads)
{
    const uint32_t id = blockIdx.x * 256u + threadIdx.x, at = divide(id, by_quads), c = (id - at * by_quads.d) * 4;     // at: row and head
    const uint32_t row = divide(at, p.by_heads), h = at - row * p.by_heads.d;
    if (row >= (uint32_t)p.q_rows || (int)row < p.q_begin[0] || (int)row >= p.q_begin[p.sequences]) return;
    const int64_t step = (int64_t)p.q_rows * p.Hq;
    const f8_f2 *ml = reinterpret_cast<const f8_f2 *>(p.partial + p.pieces * step * p.D) + at;
    float top = -__builtin_inff(), l = 0.0f;
    for (int z = 0; z < p.pieces; ++z) top = fmaxf(top, ml[z * step][0]);
    float o[4] = {0, 0, 0, 0};
    for (int z = 0; z < p.pieces; ++z) {
        const f8_f2 x = ml[z * step];
        const float w = x[0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(x[0] - top);
        float y[4];
        __builtin_memcpy(y, __builtin_assume_aligned(p.partial + (z * step + at) * p.D + c, 16), 16);
        l = fmaf(x[1], w, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(y[i], w, o[i]);
    }
    const float r = 1.0f / l;
    const uint2 y = ml[0][1] == -1.0f ? make_uint2(0, 0) : make_uint2(pair16<T>(o[0] * r, o[1] * r), pair16<T>(o[2] * r, o[3] * r));
    __builtin_memcpy(static_cast<T *>(p.o) + (int64_t)row * p.ldo + (int64_t)h * p.D + c, &y, 8);
}

// ---- host ------------------------------------------------------------------------------------------------------

template <typename T, int DP, Share SHARE>
static nq_status launch_prompt(PromptParams &p, bool direct, hipStream_t s)
{
    constexpr int TILES = 2 * stages_of(DP, SHARE) * keys_of(DP, SHARE) * pitch_of(DP) * 2, SUMS = SHARE == SHARE_KEYS ? 1024 + 2 * 64 * (DP / 2 + 1) * 4 : 0;
    constexpr int BYTES = (TILES > SUMS ? TILES : SUMS) + 16;
    p.tiles = p.q_rows / (SHARE == SHARE_ROWS ? 128 : 32) + p.sequences;
    auto launch = [&](auto kernel, std::atomic<uint64_t> &granted) {
        const nq_status st = grant_lds(kernel, BYTES, granted);
        if (st != NQ_OK) return st;
        kernel<<<dim3((unsigned)p.tiles * (unsigned)p.Hq, p.pieces), waves_of(SHARE) * 64, BYTES, s>>>(p);
        return launch_status();
    };
    static std::atomic<uint64_t> granted[3] = {};
    if constexpr (SHARE != SHARE_ALONE) {
        if (p.pieces > 1) {
            const nq_status st = launch(k_attention_prompt<T, DP, SHARE, true, true>, granted[2]);
            if (st != NQ_OK) return st;
            k_prompt_join<T><<<(unsigned)ceil_div((int64_t)p.q_rows * p.Hq * (p.D / 4), 256), 256, 0, s>>>(p, make_divider((uint32_t)p.D / 4));
            return launch_status();
        }
    }
    if constexpr (SHARE == SHARE_ALONE && DP > 128)                      // (by way of registers, of which a wave alone has too few there)
        return launch(k_attention_prompt<T, DP, SHARE, true, false>, granted[1]);
    else
        return direct ? launch(k_attention_prompt<T, DP, SHARE, true, false>, granted[1]) : launch(k_attention_prompt<T, DP, SHARE, false, false>, granted[0]);
}

// Tiles of 32 rows, whose keys the waves share, for few rows to a sequence over keys that are dealt to several workgroups, too.
static bool few_rows(int64_t sequences, int64_t q_rows, int head_dim) { return head_dim <= 128 && q_rows <= 64 * sequences; }

// Workgroups to a tile of rows, 1: it is not split.  As many as fill two to a compute unit, each with PR_LEAST keys or more, on average.  Whole and
// split, 32 heads of 128: 16 rows over 2016 keys 24.6 and 16.2 us, over 65552 753 and 88.6 (268 MB, 53 us of a copy's rate), 256 over 4256 46.1 and
// 36.7, 512 over 33280 406 and 277; 16 heads of 256, 16 rows over 32784 1260 and 98; 2 heads, 2571 causal rows 29.9 and 23.6.
constexpr int PR_LEAST = 512, PR_MOST_PIECES = 32;
static int pieces_of(int64_t sequences, int64_t q_rows, int64_t k_rows, int q_heads, int head_dim)
{
    const int64_t tiles = (ceil_div(q_rows, few_rows(sequences, q_rows, head_dim) ? 32 : 128) + sequences - 1) * q_heads;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((head_dim <= 128 ? 512 : 256) / tiles, k_rows / sequences / PR_LEAST), PR_MOST_PIECES));
}

template <typename T, int DP>
static nq_status launch_share(PromptParams &p, bool direct, hipStream_t s)
{
    const int64_t S = p.sequences, blocks = (p.q_rows / 32 + S) * p.Hq;
    if (p.pieces > 1) {
        if constexpr (DP <= 128) {
            if (few_rows(S, p.q_rows, DP)) return launch_prompt<T, DP, SHARE_KEYS>(p, direct, s);
        }
        return launch_prompt<T, DP, SHARE_ROWS>(p, direct, s);
    }
    // A wave to each 32 rows where four waves have nothing to share, or their workgroups take more than a round: sequences of up to 32 rows and 192
    // keys, on average (256 of 16 rows, 32 heads of 128, 29.8 us, 128 rows to a workgroup 113; 1000 of up to 5 91.8 and 359; 10 of up to 10, 32 heads of
    // 192, 9.0 and 14.4, but 13 rows alone, 4 heads of 256, 10.0 and 9.2), or of up to 64 rows and keys (100 of 60 43.2 and 55.0, 20 of 50 10.7 and
    // 15.0, 2 of up to 30, 8 heads, 6.0 and 7.3, but one of 33 6.8 and 6.5)
    const bool many = S * p.Hq > (DP > 128 ? 256 : 512);
    if (DP <= 128 ? (p.k_rows <= 192 * S && p.q_rows <= 32 * S && many) || (p.k_rows <= 64 * S && p.q_rows <= (S * p.Hq >= 128 ? 64 : 32) * S)
                  : p.k_rows <= 192 * S && p.q_rows <= 32 * S && many && direct)
        return launch_prompt<T, DP, SHARE_ALONE>(p, direct, s);
    // 32 rows to a workgroup and the keys dealt to its waves, where that still makes one round or two of workgroups and there are keys to deal: 512
    // rows of 32 heads 11.8 us, 128 rows to a workgroup 14.8; 1024 of 8 15.7 and 23.2; 1024 of 32 28.8 and 25.0; 64 rows over 173 keys 9.2 and 8.6; where a
    // sequence has no more than 32 rows, a round more: 16 of up to 16 over up to 2000 keys 32.0 and 41.0
    if constexpr (DP <= 128) {
        if (blocks <= (p.q_rows <= 32 * S ? 1024 : 576) && p.k_rows >= 192 * S) return launch_prompt<T, DP, SHARE_KEYS>(p, direct, s);
    }
    return launch_prompt<T, DP, SHARE_ROWS>(p, direct, s);
}

template <typename T>
static nq_status run_prompt(PromptParams &p, bool direct, hipStream_t s)
{
    if (p.D <= 64) return launch_share<T, 64>(p, direct, s);
    if (p.D <= 96) return launch_share<T, 96>(p, direct, s);
    if (p.D <= 128) return launch_share<T, 128>(p, direct, s);
    if (p.D <= 192) return launch_share<T, 192>(p, direct, s);
    return launch_share<T, 256>(p, direct, s);
}

}  // namespace nq

using namespace nq;

extern "C" size_t nq_attention_prompt_workspace_bytes(int64_t sequences, int64_t q_rows, int64_t k_rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    if (sequences < 1 || q_rows < 1 || k_rows < 1 || sequences > ATT_MAX_ROWS || q_rows > ATT_MAX_ROWS || k_rows > ATT_MAX_ROWS) return 0;
    if (check_heads(q_heads, kv_heads, head_dim) != NQ_OK || q_heads % kv_heads) return 0;
    const int pieces = pieces_of(sequences, q_rows, k_rows, q_heads, head_dim);
    return pieces > 1 ? (size_t)pieces * q_rows * q_heads * (head_dim + 2) * sizeof(float) : 0;
}

extern "C" nq_status nq_attention_prompt(const nq_prompt_job *job, void *stream)
{
    if (!job || job->sequences < 0 || job->q_rows < 0 || job->k_rows < 0) return NQ_ERR_INVALID_ARG;
    const nq_prompt_job &j = *job;
    if (!is_dtype(j.dtype)) return NQ_ERR_INVALID_ARG;
    nq_status st;
    if ((st = check_heads(j.q_heads, j.kv_heads, j.head_dim)) != NQ_OK) return st;
    if (j.q_heads % j.kv_heads) return NQ_ERR_SHAPE;
    if (j.dtype == NQ_DT_F32) return NQ_ERR_UNSUPPORTED;
    if (j.q_rows > ATT_MAX_ROWS || j.k_rows > ATT_MAX_ROWS || j.sequences > ATT_MAX_ROWS) return NQ_ERR_SHAPE;
    // (a dispatch has fewer than 2^32 threads)
    if ((j.q_rows / 128 + j.sequences) * j.q_heads >= (int64_t(1) << 24)) return NQ_ERR_SHAPE;
    if (j.sequences == 0 || j.q_rows == 0) return NQ_OK;
    const int64_t wq = (int64_t)j.q_heads * j.head_dim, wk = (int64_t)j.kv_heads * j.head_dim;
    if ((st = check_matrix(j.d_q, j.dtype, wq, j.ldq)) != NQ_OK) return st;
    if ((st = check_matrix(j.d_o, j.dtype, wq, j.ldo)) != NQ_OK) return st;
    if (j.k_rows > 0 && (st = check_matrix(j.d_k, j.dtype, wk, j.ldk)) != NQ_OK) return st;
    if (j.k_rows > 0 && (st = check_matrix(j.d_v, j.dtype, wk, j.ldv)) != NQ_OK) return st;
    if (!j.d_q_begin) return NQ_ERR_INVALID_ARG;
    if (!aligned_to(j.d_q_begin, 4) || !aligned_to(j.d_k_begin, 4)) return NQ_ERR_ALIGN;

    PromptParams p;
    p.q = j.d_q;
    p.k = j.d_k;
    p.v = j.d_v;
    p.o = j.d_o;
    p.q_begin = j.d_q_begin;
    p.k_begin = j.d_k_begin ? j.d_k_begin : j.d_q_begin;
    p.ldq = j.ldq;
    p.ldk = j.ldk;
    p.ldv = j.ldv;
    p.ldo = j.ldo;
    p.sequences = (int32_t)j.sequences;
    p.q_rows = (int32_t)j.q_rows;
    p.k_rows = (int32_t)j.k_rows;
    p.Hq = j.q_heads;
    p.Hkv = j.kv_heads;
    p.group = j.q_heads / j.kv_heads;
    p.D = j.head_dim;
    p.causal = j.causal != 0;
    p.by_heads = make_divider((uint32_t)j.q_heads);
    p.scale = j.scale == 0.0f ? 1.0f : j.scale < 0.0f ? -j.scale * PR_LOG2E : j.scale * PR_LOG2E;
    p.flip = j.scale < 0.0f ? 0x80008000u : 0u;
    p.zero = j.scale == 0.0f;
    p.first_half = std::max(1, 256 / j.q_heads);
    // rows on 16 bytes, a tile's offsets within 31 bits
    const bool direct = aligned16(j.d_q) && aligned16(j.d_k) && aligned16(j.d_v) && j.ldq % 8 == 0 && j.ldk % 8 == 0 && j.ldv % 8 == 0 &&
                        std::max(std::max(j.ldq, j.ldk), j.ldv) < (int64_t(1) << 23);
    p.partial = static_cast<float *>(j.d_workspace);
    p.pieces = 1;
    if (j.d_workspace) {
        if (!aligned16(j.d_workspace)) return NQ_ERR_ALIGN;
        if (j.workspace_bytes < nq_attention_prompt_workspace_bytes(j.sequences, j.q_rows, j.k_rows, j.q_heads, j.kv_heads, j.head_dim)) return NQ_ERR_RANGE;
        // (rows that are not on 16 bytes: not split)
        if (direct && j.k_rows > 0) p.pieces = pieces_of(j.sequences, j.q_rows, j.k_rows, j.q_heads, j.head_dim);
    }
    return j.dtype == NQ_DT_F16 ? run_prompt<_Float16>(p, direct, (hipStream_t)stream) : run_prompt<bf16_t>(p, direct, (hipStream_t)stream);
}
