// Attention over the 4-bit key/value cache.
//
// For query row n and tokens j: x_j = scale s_j (q_n . K_j), out = sum_j 2^(x_j log2 e - m) s'_j V_j / sum_j 2^(x_j log2 e - m),
// K_j and V_j rows of levels, s_j and s'_j the rows' scales.  A wave keeps 16 * NT query rows (a row: one head of the
// group at one query token) and takes 32 tokens a step; maximum, sum and the products with the values stay in
// registers over all steps.
//
// Scores are S^T = K q^T by 16x16x32 MFMA: rows are 16 tokens, columns query rows.  The wave's 64 lanes are 16 columns
// (n = lane % 16) by 4 quarters (q = lane / 16); an operand's 8 reduction elements of a lane are 8 channels of one token, one dword of
// codes.  Which channels is free as long as q agrees, so quarter q takes the contiguous channels [q d/4, (q+1) d/4) of its
// token.  A lane receives the scores of tokens 4q .. 4q+3 of its column, for two 16-token halves: 8 weights, which
// are the 8 reduction elements of the operand w^T of O^T = V^T w^T as they stand, since a sum over tokens takes them in any
// order.  The operand V^T holds for one channel the levels of these 8 tokens: dwords of codes of two tokens are interleaved by half
// bytes (one v_bfi), so that each byte again holds two codes that the product wants side by side.
//
// Codes become levels two at a time: a byte is the index into a table of 256 pairs of 16-bit levels in LDS, held 32 times, one copy a
// bank, so that a wave's 64 random indices do not collide.  A row of the table is 256 bytes, the keys' copies in the lower half and the
// values' in the upper: the address is (byte << 8) + 4 (lane % 32) + 128 for values, one v_perm and an offset in the instruction.  Values
// are multiplied as fp16 whatever t is (levels are at most 1 or so, 11 bits hold a bf16's 8).
//
// The running maximum is only moved when a score passes it by 2^kSlack, the weights' scale (a power of two near the largest s') when one
// passes that by 2^kScaleSlack: the sums are then multiplied once.  Weights stay below 2^15 and fit fp16.
#include <algorithm>

#include "fk_device.h"
#include "fk_kv.h"

namespace fk {

constexpr float kSlack = 8.f;            // in powers of two
constexpr float kScaleSlack = 64.f;
constexpr float kNone = -3.402823466e38f;  // maximum of a row that has seen nothing
constexpr int kJoinWaves = 8;            // waves of a workgroup that share the rows
constexpr int kOwnWaves = 4;             // waves of a workgroup with rows of their own
constexpr int kStep = 32;                // tokens a wave takes at a time
constexpr size_t kTableBytes = 65536;
constexpr int kMostSplits = 256;          // of one row block's tokens
constexpr int kPagesAhead = 32;          // steps whose pages a wave holds in one register (two halves each)

template <bool BF>
__device__ __forceinline__ floatx4 mfma16(uintx4 a, uintx4 b, floatx4 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t float_to_half(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    return float_to_half(lo) | float_to_half(hi) << 16;
}

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// kScaleSlack units as two numbers of type t, at most the largest finite one
template <bool BF>
__device__ __forceinline__ uint32_t limit_of(float unit) {
    const uint32_t l = float_to_lp_any(fminf(kScaleSlack * unit, BF ? 0x1.fep127f : 65504.f), BF);
    return l | l << 16;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

struct AttendArgs {
    KVView c;
    KVAttend a;
    int group;                 // query heads to a cache head
    int splits, row_blocks;
    int chunk;
    float scale_log2;          // positive, so that scores that are not seen stay -inf:
    uint32_t flip;             // the signs of the queries' channels are flipped instead
};

// Blocks of the values' channels by the number of bytes that a lane takes of each: ND bytes in pieces of 4, 2 and 1 (powers of two, so
// that the loads are aligned).  Piece p starts at byte 16 * (bytes before it) of the row.
template <int ND> struct Pieces {
    static constexpr int whole = ND / 4, two = (ND & 2) ? 1 : 0, one = ND & 1;
    static constexpr int count = whole + two + one;
    static constexpr int width(int p) { return p < whole ? 4 : p < whole + two ? 2 : 1; }
    static constexpr int before(int p) { return p < whole ? 4 * p : p < whole + two ? 4 * whole : 4 * whole + 2 * two; }
};

template <int ND> struct Codes {
    uint32_t k[2][ND];                     // keys of token (lane % 16) of either half
    uint32_t v[2][4][Pieces<ND>::count];   // values of tokens 4q + r
    uintx2 ks[2], vs[2];                   // scales of tokens 4q .. 4q+3, 16 bits each
};

// Channel of O^T's row m of subtile s (s = piece byte and half)
template <int ND>
__device__ __forceinline__ int channel_of(int s, int m) {
    using P = Pieces<ND>;
    const int byte = s / 2;
    int p = 0;
#pragma unroll
    for (int i = 1; i < P::count; ++i) p = byte >= P::before(i) ? i : p;
    return 2 * (16 * P::before(p) + m * P::width(p) + (byte - P::before(p))) + (s & 1);
}

template <bool BF, int ND>
struct Reader {
    const AttendArgs& A;
    const int32_t* table;      // the sequence's pages
    int h, last_half;          // cache head; start of the last 16 tokens that are read
    int lane, n, q;

    // page of the 16 tokens from `at`, or of the last ones where that is past the end
    __device__ __forceinline__ int page_of(int at) const {
        const int p = table[min(at, last_half) >> A.c.page_shift];
        return min(max(p, 0), (int)A.c.pages - 1);
    }

    // first rows of a step's halves
    __device__ __forceinline__ void rows_of(int64_t (&row)[2], int at, int page0, int page1) const {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int from = min(at + 16 * u, last_half) & ((1 << A.c.page_shift) - 1);
            row[u] = (((int64_t)(u ? page1 : page0) * A.c.heads + h) << A.c.page_shift) + from;
        }
    }
    // (bases are the same in all lanes, what differs between lanes is an unsigned 32-bit offset: one address register for all loads
    // of a kind)
    __device__ __forceinline__ void load_keys(Codes<ND>& f, const int64_t (&row)[2]) const {
        const uint32_t of = n * (16 * ND) + q * (4 * ND);
#pragma unroll
        for (int u = 0; u < 2; ++u) __builtin_memcpy(f.k[u], __builtin_assume_aligned(A.c.k_codes + row[u] * (16 * ND) + of, 4), 4 * ND);
    }
    __device__ __forceinline__ void load_scales(Codes<ND>& f, const int64_t (&row)[2]) const {
        const uint32_t of = 8 * q;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f.ks[u] = *(const uintx2*)((const uint8_t*)(A.c.k_scale + row[u]) + of);
            f.vs[u] = *(const uintx2*)((const uint8_t*)(A.c.v_scale + row[u]) + of);
        }
    }
    __device__ __forceinline__ void load_values(Codes<ND>& f, const int64_t (&row)[2]) const {
        using P = Pieces<ND>;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int p = 0; p < P::count; ++p) {
                const uint32_t of = q * 4 * (16 * ND) + n * P::width(p);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint8_t* at = A.c.v_codes + row[u] * (16 * ND) + of + (r * (16 * ND) + 16 * P::before(p));
                    f.v[u][r][p] = P::width(p) == 4 ? *(const uint32_t*)at : P::width(p) == 2 ? *(const uint16_t*)at : *at;
                }
            }
    }
};

template <bool BF>
__device__ __forceinline__ float scale_at(uintx2 s, int r) { return lp_to_float((uint16_t)(s[r / 2] >> 16 * (r & 1)), BF); }

// Two levels of each of four bytes: byte b of the words, in order
template <int OFFSET>
__device__ __forceinline__ uint32_t pair_of(const uint8_t* lds, uint32_t word, int b, uint32_t copy) {
    return *(const uint32_t*)(lds + __builtin_amdgcn_perm(word, copy, 0x0c0c0400u | (uint32_t)b << 8) + OFFSET);
}

template <bool BF, int ND, int NT, bool JOIN>
__global__ __launch_bounds__(64 * (JOIN ? kJoinWaves : kOwnWaves), JOIN && NT == 1 && ND <= 4 ? 4 : 1) void kv_attend_kernel(AttendArgs A) {
    // (a fixed size, so that the compiler knows the table's address and leaves it to the instruction's offset)
    __shared__ __align__(16) uint8_t lds[kTableBytes + (JOIN ? 2 * kJoinWaves * 16 * NT * 4 : 0)];
    using P = Pieces<ND>;
    constexpr int R = 16 * NT, S = 2 * ND, W = JOIN ? kJoinWaves : 1, THREADS = 64 * (JOIN ? kJoinWaves : kOwnWaves);
    const int b = blockIdx.z, h = blockIdx.y, split = blockIdx.x % A.splits, rb = blockIdx.x / A.splits;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const KVAttend& a = A.a;

    const int len = min(max(a.lens[b], 0), a.max_pages << A.c.page_shift);
    const int q0 = a.q_start ? min(max(a.q_start[b], 0), (int)a.Tq) : b * a.max_q;
    const int nq = a.q_start ? min(min(max(a.q_start[b + 1] - q0, 0), a.max_q), (int)a.Tq - q0) : a.max_q;
    const int rows = nq * A.group;
    const int row0 = (JOIN ? rb : rb * kOwnWaves + wave) * R;
    if ((JOIN ? row0 : rb * kOwnWaves * R) >= rows) return;       // the whole workgroup

    // tokens that the wave's rows see
    const int i0 = row0 / A.group, i1 = (min(row0 + R, rows) - 1) / A.group;
    const int p0 = len - nq + i0, p1 = len - nq + i1;
    const int hi = row0 >= rows ? 0 : a.causal ? max(min(len, p1 + 1), 0) : len;
    const int lo = a.window ? max(0, p0 - a.window + 1) : 0;
    const int first = (lo & ~(kStep - 1)) + split * A.chunk;
    const int end = split == A.splits - 1 ? hi : min(hi, first + A.chunk);
    if (JOIN && split > 0 && first >= hi) return;                 // the whole workgroup
    // a step is whole where every row sees all of its tokens
    const int whole_end = a.causal ? min(len, p0 + 1) : len, whole_from = a.window ? p1 - a.window + 1 : 0;
    const int mine = first + (JOIN ? wave * kStep : 0);
    const int steps = end > mine ? (end - mine + W * kStep - 1) / (W * kStep) : 0;

    Reader<BF, ND> in{A, a.pages + (int64_t)b * a.max_pages, h, max(hi - 1, 0) & ~15, lane, n, q};
    int ahead = 0;                                                // lane l: page of half l % 2 of step l / 2 of this batch
    auto pages_from = [&](int step) { return in.page_of(mine + (step + lane / 2) * W * kStep + (lane & 1) * 16); };
    Codes<ND> f;                                                  // the step's, refilled piece by piece as it is used up
    int64_t row[2];
    if (steps) {
        ahead = pages_from(0);
        in.rows_of(row, mine, __builtin_amdgcn_readlane(ahead, 0), __builtin_amdgcn_readlane(ahead, 1));
        in.load_keys(f, row);
        in.load_scales(f, row);
        in.load_values(f, row);
    }

    {   // The table of pairs.  Lanes 0..15 hold the keys' levels, lanes 16..31 the values'; sixteen pieces of 16 bytes make a row.
        const uint16_t level = ((lane & 16) ? A.c.v_levels : A.c.k_levels)[h * 16 + (lane & 15)];
        const uint32_t mine = (lane & 16) ? float_to_half(lp_to_float(level, BF)) : level;
        const int side = (lane & 8) * 2;
#pragma unroll
        for (int i = 0; i < (int)kTableBytes / 16 / THREADS; ++i) {
            const int at = i * THREADS + threadIdx.x, code = at / 16;
            const uint32_t pair = (uint32_t)__shfl((int)mine, side + (code & 15)) | ((uint32_t)__shfl((int)mine, side + (code >> 4)) << 16);
            ((uintx4*)lds)[at] = uintx4{pair, pair, pair, pair};
        }
    }

    // query rows: operand, and the tokens that each column's row sees
    uintx4 Q[NT][ND];
    int see_lo[NT], see_hi[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const int row = row0 + c * 16 + n, i = row / A.group, g = row - i * A.group;
        const bool live = row < rows;
        const uint16_t* at = a.q.at + (int64_t)(q0 + i) * a.q.token + (int64_t)(h * A.group + g) * a.q.head + q * (8 * ND);
#pragma unroll
        for (int k = 0; k < ND; ++k) {
            Q[c][k] = uintx4{0, 0, 0, 0};
            if (live) Q[c][k] = *(const uintx4_any*)(at + 8 * k) ^ A.flip;
        }
        const int pos = len - nq + i;
        see_hi[c] = !live ? 0 : a.causal ? min(len, pos + 1) : len;
        see_lo[c] = a.window ? pos - a.window + 1 : 0;
    }

    floatx4 O[S][NT];
    float top[NT], sum[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        top[c] = kNone;
        sum[c] = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) O[s][c] = floatx4{0, 0, 0, 0};
    }
    float unit = 0.f, per_unit = 1.f;                             // of the weights: a power of two near the largest s'
    uint32_t limit2 = 0;                                          // kScaleSlack units as type t, twice
    const uint32_t copy = (lane & 31) * 4;
    __syncthreads();

    for (int it = 0; it < steps; ++it) {
        const int at = mine + it * W * kStep;
        if ((it + 1) % kPagesAhead == 0) ahead = pages_from(it + 1);
        const int l = 2 * ((it + 1) % kPagesAhead);
        // rows of the next step (after the last one: of the sequence's end, not used)
        in.rows_of(row, at + W * kStep, __builtin_amdgcn_readlane(ahead, l), __builtin_amdgcn_readlane(ahead, l + 1));

        floatx4 X[2][NT];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < NT; ++c) X[u][c] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < ND; ++k) {
                uintx4 op;
#pragma unroll
                for (int j = 0; j < 4; ++j) op[j] = pair_of<0>(lds, f.k[u][k], j, copy);
#pragma unroll
                for (int c = 0; c < NT; ++c) X[u][c] = mfma16<BF>(op, Q[c][k], X[u][c]);
            }
        in.load_keys(f, row);

        float vs[8], x[NT][8], peak[NT];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            vs[e] = scale_at<BF>(f.vs[e / 4], e & 3);
#pragma unroll
            for (int c = 0; c < NT; ++c) x[c][e] = X[e / 4][c][e & 3] * scale_at<BF>(f.ks[e / 4], e & 3);
        }
        if (at + kStep > whole_end || at < whole_from) {          // some row does not see all of these tokens
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int token = at + 4 * q + 16 * (e / 4) + (e & 3);
                // A scale that is not finite reaches the rows that see it by way of their scores; where none does, or the tokens are
                // past the end, it may be anything.
                const bool bad = !(vs[e] <= 3.402823466e38f);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    x[c][e] = token < see_lo[c] || token >= see_hi[c] ? -INFINITY : bad ? NAN : x[c][e];
                if (bad || token < lo || token >= hi) vs[e] = 0.f;
            }
        }
        // The largest scale of the values against the limit, two at a time as 16-bit integers (they are positive), and the scores
        // against the maxima.
        uint32_t most2 = limit2;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 2; ++j) most2 = pk_max_u16(most2, f.vs[u][j]);
        in.load_scales(f, row);
        bool move = most2 != limit2;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            peak[c] = kNone;
#pragma unroll
            for (int e = 0; e < 8; ++e) peak[c] = fmaxf(peak[c], x[c][e]);
            move |= fmaf(peak[c], A.scale_log2, -top[c]) > kSlack;
        }
        if (__any(move)) {
            float most = 0.f, ratio = 1.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, vs[e]);
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            if (most > kScaleSlack * unit) {                      // the same in all lanes
                const float to = fminf(__uint_as_float(max(__float_as_uint(most) & 0x7f800000u, 0x00800000u)), 0x1p126f);
                ratio = unit / to;
                unit = to;
                per_unit = 1.f / to;
                limit2 = limit_of<BF>(unit);
            }
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                float to = fmaxf(peak[c], __shfl_xor(peak[c], 16));
                to = fmaxf(to, __shfl_xor(to, 32));
                // (a column's maximum moves by its own scores alone: what other rows see has no part in its rounding)
                to = fmaf(to, A.scale_log2, -top[c]) > kSlack ? to * A.scale_log2 : top[c];
                const float shrink = exp2_fast(top[c] - to);
                top[c] = to;
                sum[c] *= shrink;
#pragma unroll
                for (int s = 0; s < S; ++s) O[s][c] *= shrink * ratio;
            }
        }
        uintx4 w[NT];
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] *= per_unit;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[c][e] = exp2_fast(fmaf(x[c][e], A.scale_log2, -top[c]));
                sum[c] += x[c][e];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) w[c][j] = pack_half2(x[c][2 * j] * vs[2 * j], x[c][2 * j + 1] * vs[2 * j + 1]);
        }

#pragma unroll
        for (int p = 0; p < P::count; ++p) {
            uint32_t pairs[4][2];                                 // [two tokens][half byte]
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w0 = f.v[j / 2][2 * (j & 1)][p], w1 = f.v[j / 2][2 * (j & 1) + 1][p];
                pairs[j][0] = (w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u);
                pairs[j][1] = ((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u);
            }
#pragma unroll
            for (int i = 0; i < P::width(p); ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uintx4 op;
#pragma unroll
                    for (int j = 0; j < 4; ++j) op[j] = pair_of<128>(lds, pairs[j][half], i, copy);
                    const int s = 2 * (P::before(p) + i) + half;
#pragma unroll
                    for (int c = 0; c < NT; ++c) O[s][c] = mfma16<false>(op, w[c], O[s][c]);
                }
        }
        in.load_values(f, row);
    }

#pragma unroll
    for (int c = 0; c < NT; ++c) {
        sum[c] += __shfl_xor(sum[c], 16);
        sum[c] += __shfl_xor(sum[c], 32);
#pragma unroll
        for (int s = 0; s < S; ++s) O[s][c] *= unit;
    }

    const bool partial = A.splits > 1 && (hi - (lo & ~(kStep - 1))) > A.chunk;
    float* part = a.part + ((((int64_t)b * A.c.heads + h) * A.row_blocks + rb) * A.splits + split) * (R * (32 * ND + 2));
    auto finish = [&](int c, int s, floatx4 o, float t, float l) {
        const int row = row0 + c * 16 + n, i = row / A.group, g = row - i * A.group;
        if (row >= rows) return;
        const int64_t at = (int64_t)(q0 + i) * a.q_heads + h * A.group + g;
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) a.out[at * (32 * ND) + channel_of<ND>(s, 4 * q + r)] = float_to_lp_any(o[r] * inv, BF);
        if (a.lse && s == 0 && q == 0) a.lse[at] = l > 0.f || l != l ? (t + __log2f(l)) * 0.6931471805599453f : -INFINITY;
    };

    if constexpr (!JOIN) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int s = 0; s < S; ++s) finish(c, s, O[s][c], top[c], sum[c]);
    } else {
        // The waves' maxima and sums, then their products by way of the table's memory, a few subtiles at a time.
        float* tops = (float*)(lds + kTableBytes);                // [waves][R]
        float* sums = tops + kJoinWaves * R;
        if (q == 0)
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                tops[wave * R + c * 16 + n] = sum[c] == 0.f ? kNone : top[c];
                sums[wave * R + c * 16 + n] = sum[c];
            }
        __syncthreads();                                          // the table is done with, too
        float t[NT], l[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            t[c] = kNone;
            l[c] = 0.f;
            for (int w = 0; w < kJoinWaves; ++w) t[c] = fmaxf(t[c], tops[w * R + c * 16 + n]);
            for (int w = 0; w < kJoinWaves; ++w) l[c] += sums[w * R + c * 16 + n] * exp2_fast(tops[w * R + c * 16 + n] - t[c]);
            const float mine = sum[c] == 0.f ? 0.f : exp2_fast(top[c] - t[c]);
#pragma unroll
            for (int s = 0; s < S; ++s) O[s][c] *= mine;
        }
        constexpr int AT_ONCE = (int)(kTableBytes / 16) / (64 * kJoinWaves * NT);
        static_assert(AT_ONCE >= 1, "the joined products fit the table's memory");
        floatx4* swap = (floatx4*)lds;                            // [waves][AT_ONCE][NT][64]
#pragma unroll
        for (int s0 = 0; s0 < S; s0 += AT_ONCE) {
            if (s0) __syncthreads();
#pragma unroll
            for (int s = s0; s < s0 + AT_ONCE && s < S; ++s)
#pragma unroll
                for (int c = 0; c < NT; ++c) swap[((wave * AT_ONCE + s - s0) * NT + c) * 64 + lane] = O[s][c];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < AT_ONCE * NT; k += kJoinWaves) {  // (subtile, column tile) of this wave
                const int i = k + wave, c = i % NT, s = s0 + i / NT;
                if (i >= AT_ONCE * NT || s >= S) continue;
                floatx4 o = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < kJoinWaves; ++w) o += swap[(w * AT_ONCE * NT + i) * 64 + lane];
                float tc = t[0], lc = l[0];
#pragma unroll
                for (int j = 1; j < NT; ++j) { tc = c == j ? t[j] : tc; lc = c == j ? l[j] : lc; }
                if (partial) {
                    if (row0 + c * 16 + n >= rows) continue;
                    ((floatx4*)(part + 2 * R))[(s * NT + c) * 64 + lane] = o;
                    if (s == 0 && q == 0) {
                        part[c * 16 + n] = tc;
                        part[R + c * 16 + n] = lc;
                    }
                } else {
                    finish(c, s, o, tc, lc);
                }
            }
        }
    }
}

// Joins the splits of one subtile of one row block.  All their maxima and sums are read at once, 16 columns by 32 splits, and become the
// splits' factors in LDS; then each of the eight waves adds every eighth split's products, and the first wave what they have.
constexpr int kJoinThreads = 512;
template <bool BF, int ND, int NT>
__global__ __launch_bounds__(kJoinThreads) void kv_join_kernel(AttendArgs A) {
    constexpr int R = 16 * NT, WAVES = kJoinThreads / 64, LANES = kJoinThreads / 16;
    __shared__ floatx4 swap[WAVES][64];
    __shared__ float factor[kMostSplits][16], most[WAVES][16], all[WAVES][16];
    const KVAttend& a = A.a;
    const int b = blockIdx.z, h = blockIdx.y, tile = blockIdx.x % (2 * ND * NT), rb = blockIdx.x / (2 * ND * NT);
    const int s = tile / NT, c = tile % NT;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int len = min(max(a.lens[b], 0), a.max_pages << A.c.page_shift);
    const int q0 = a.q_start ? min(max(a.q_start[b], 0), (int)a.Tq) : b * a.max_q;
    const int nq = a.q_start ? min(min(max(a.q_start[b + 1] - q0, 0), a.max_q), (int)a.Tq - q0) : a.max_q;
    const int rows = nq * A.group, row0 = rb * R;
    if (row0 + c * 16 >= rows) return;
    const int i0 = row0 / A.group, i1 = (min(row0 + R, rows) - 1) / A.group;
    const int hi = a.causal ? max(min(len, len - nq + i1 + 1), 0) : len;
    const int lo = (a.window ? max(0, len - nq + i0 - a.window + 1) : 0) & ~(kStep - 1);
    if (hi - lo <= A.chunk) return;                               // one split has written the result itself
    const int parts = min(A.splits, (hi - lo + A.chunk - 1) / A.chunk);
    const int64_t stride = R * (32 * ND + 2);
    const float* part = a.part + (((int64_t)b * A.c.heads + h) * A.row_blocks + rb) * A.splits * stride;
    const int col = c * 16 + n;
    const bool live = row0 + col < rows;

    constexpr int EACH = kMostSplits / LANES;
    float tops[EACH], sums[EACH], t = kNone, l = 0.f;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int i = k * LANES + wave * 4 + q;
        tops[k] = i < parts && live ? part[i * stride + col] : kNone;
        sums[k] = i < parts && live ? part[i * stride + R + col] : 0.f;
        t = fmaxf(t, tops[k]);
    }
    t = fmaxf(t, __shfl_xor(t, 16));
    t = fmaxf(t, __shfl_xor(t, 32));
    if (q == 0) most[wave][n] = t;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t = fmaxf(t, most[w][n]);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const float f = exp2_fast(tops[k] - t);
        factor[k * LANES + wave * 4 + q][n] = f;
        l += sums[k] * f;
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (q == 0) all[wave][n] = l;
    __syncthreads();

    floatx4 o = {0, 0, 0, 0};
    const floatx4* from = (const floatx4*)(part + 2 * R) + (s * NT + c) * 64 + lane;
    if (live)
#pragma unroll 8
        for (int i = wave; i < parts; i += WAVES) o += factor[i][n] * *(const floatx4*)((const float*)from + i * stride);
    swap[wave][lane] = o;
    __syncthreads();
    if (wave || !live) return;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) l += all[w][n];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) o += swap[w][lane];
    const int row = row0 + col, i = row / A.group, g = row - i * A.group;
    const int64_t at = (int64_t)(q0 + i) * a.q_heads + h * A.group + g;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) a.out[at * (32 * ND) + channel_of<ND>(s, 4 * q + r)] = float_to_lp_any(o[r] * inv, BF);
    if (a.lse && s == 0 && q == 0) a.lse[at] = l > 0.f || l != l ? (t + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

KVPlan choose_kv_plan(const KVView& c, int q_heads, int B, int max_q, int64_t reach) {
    const int group = q_heads / c.heads;
    const int64_t rows = (int64_t)max_q * group;
    const int most = c.d <= 128 ? 4 : 2;                         // tiles of a wave
    KVPlan p;
    p.join = rows <= 16 * most || (int64_t)B * c.heads * cdiv(rows, 16 * most * kOwnWaves) < device_cu_count();
    p.tiles = !p.join ? most : rows <= 16 ? 1 : rows <= 32 ? 2 : most;
    p.row_blocks = (int)cdiv(rows, 16 * p.tiles * (p.join ? 1 : kOwnWaves));
    p.splits = 1;
    p.chunk = INT32_MAX / 2;
    if (p.join) {
        const int64_t wg = kJoinWaves * kStep, slots = (int64_t)device_cu_count() * 2, blocks = (int64_t)B * c.heads * p.row_blocks;
        const int64_t want = blocks >= slots ? 1 : slots / blocks, steps = cdiv(reach, wg);
        p.splits = (int)std::min({want, steps, (int64_t)kMostSplits});
        if (p.splits > 1) p.chunk = cdiv(steps, p.splits) * wg;
    }
    return p;
}

template <bool BF, int ND, int NT, bool JOIN>
static fk_status launch_form(const AttendArgs& A, hipStream_t s) {
    const int waves = JOIN ? kJoinWaves : kOwnWaves;
    kv_attend_kernel<BF, ND, NT, JOIN><<<dim3(A.row_blocks * A.splits, A.c.heads, A.a.B), 64 * waves, 0, s>>>(A);
    FK_HIP(hipGetLastError());
    if (JOIN && A.splits > 1) {
        kv_join_kernel<BF, ND, NT><<<dim3(A.row_blocks * 2 * ND * NT, A.c.heads, A.a.B), kJoinThreads, 0, s>>>(A);
        FK_HIP(hipGetLastError());
    }
    return FK_OK;
}

template <bool BF, int ND>
static fk_status launch_width(const AttendArgs& A, const KVPlan& p, hipStream_t s) {
    if (!p.join) return launch_form<BF, ND, (ND <= 4 ? 4 : 2), false>(A, s);
    if (p.tiles == 1) return launch_form<BF, ND, 1, true>(A, s);
    if (p.tiles == 2) return launch_form<BF, ND, 2, true>(A, s);
    if constexpr (ND <= 4) return launch_form<BF, ND, 4, true>(A, s);
    set_error("fk_kv_attend: no form of %d tiles for d=%d", p.tiles, 32 * ND);
    return FK_EUNSUPPORTED;
}

template <bool BF>
static fk_status launch_type(const AttendArgs& A, const KVPlan& p, hipStream_t s) {
    switch (A.c.d / 32) {
        case 1: return launch_width<BF, 1>(A, p, s);
        case 2: return launch_width<BF, 2>(A, p, s);
        case 3: return launch_width<BF, 3>(A, p, s);
        case 4: return launch_width<BF, 4>(A, p, s);
        case 5: return launch_width<BF, 5>(A, p, s);
        case 6: return launch_width<BF, 6>(A, p, s);
        case 7: return launch_width<BF, 7>(A, p, s);
        default: return launch_width<BF, 8>(A, p, s);
    }
}

fk_status launch_kv_attend(const KVView& c, const KVAttend& a, const KVPlan& p, hipStream_t s) {
    const AttendArgs A{c, a, a.q_heads / c.heads, p.splits, p.row_blocks, (int)p.chunk, fmaxf(fabsf(a.scale) * 1.44269504088896341f, 1e-37f), a.scale < 0.f ? 0x80008000u : 0u};
    return c.bf ? launch_type<true>(A, p, s) : launch_type<false>(A, p, s);
}

}  // namespace fk
