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
// are multiplied as fp16 whatever t is; levels of bf16 times the power of two that puts the head's largest at 2^14, so that those down to
// 2^-31 of it keep their 8 bits, and the products are divided by it at the end.
//
// The exponents' reference m of a row follows its weights 2^(x_j log2 e - m) s'_j rather than its scores: a row's largest weight is put
// at 2^kTop, and the reference is only moved, and the sums multiplied once, when a weight would pass 2^kFits.  So the weights, which are
// multiplied as fp16, keep 11 bits, as many as the values have in an uncoded cache of fp16, down to 2^-20 of the row's largest, and
// vanish below 2^-31 of it, whatever scales other rows see.  The exponentials' sums and the statistics are fp32; where scales are so small
// that exponentials would pass 2^kMost, weights stay smaller instead.
//
// What bounds it.  Single tokens (at most 16 query rows to a cache head): bytes, 2 (d/2 + 2) a token and head.  64 sequences of up to 8192
// tokens, 8 heads of 128: 353 MB in 83 us, 4.2 TB/s (5.0 where they are equally long; a large copy reaches 5.2); one of 131072: 138 MB in 31
// to 34 us and the join 4.9.  Few tokens: a workgroup's fixed cost, about 6 us with its launch, of which the chain of first loads (page, codes; the length
// is not waited for), the table (64 KiB of LDS) and the exchange between the waves are a third each, then 1.1 us a step of 8 x 32 tokens.
// Many sequences of few tokens share workgroups, a wave each: 110 of up to 9, 9 heads, 7.6 us.
// Many rows: vector instructions.  A step of 48 rows and 32 tokens at d = 128 takes 48 MFMA (768 cycles), 64 lookups and about 240 vector
// instructions with 24 exponentials (1340 cycles); two waves a SIMD overlap a third of the two.  Two sequences of 4096 queries over up to
// 9000 tokens, 32 query heads: 852 GFLOP in 1058 us, 0.8 PFLOP/s (the first 30 passes of a program 1130); a large product of the library reaches 1.2 on this card.
#include <algorithm>

#include "fk_device.h"
#include "fk_kv.h"

namespace fk {

// Weights, in powers of two: the largest after its reference has moved, and at any time.  (The chunk named above: 2^8 1078 us, 2^6 1060, 2^3 1055,
// since references move less often; each of them drops one more power of two of the smallest weights.)
constexpr float kTop = 6.f, kFits = 15.5f;
constexpr float kMost = 96.f, kMostMoved = 90.f;   // the same for the exponentials, of which up to 2^30 are added up
constexpr float kNone = -3.402823466e38f;   // below every score: the maximum of a row that has seen nothing
constexpr int kJoinWaves = 8;            // waves of a workgroup that share the rows
constexpr int kStep = 32;                // tokens a wave takes at a time
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
// two products rounded to fp16, each by the instruction that multiplies
__device__ __forceinline__ uint32_t pack_products(float a, float b, float c, float d) {
    typedef _Float16 half2v __attribute__((ext_vector_type(2)));
    half2v r;
    r[0] = (_Float16)(a * b);
    r[1] = (_Float16)(c * d);
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// x 2^by for by below 0, of which 2^by alone may be too small for 32 bits
__device__ __forceinline__ float times_exp2(float x, float by) {
    const float half = exp2_fast(0.5f * by);
    return x * half * half;
}

// x / by for any x below 2^32: a multiplication by 2^(32 + s) / by, s = ceil(log2 by), less 2^32
struct Divider {
    int by;
    uint32_t factor;
    int shift1, shift2;
    explicit Divider(int d) : by(d) {
        int s = 0;
        while (s < 31 && (1 << s) < d) ++s;
        factor = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - d)) / d + 1);
        shift1 = s ? 1 : 0;
        shift2 = s ? s - 1 : 0;
    }
    __device__ __forceinline__ int quotient(int x) const {
        const uint32_t t = __umulhi((uint32_t)x, factor);
        return (int)((t + (((uint32_t)x - t) >> shift1)) >> shift2);
    }
};

struct AttendArgs {
    KVView c;
    KVAttend a;
    Divider group;             // query heads to a cache head
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

// An address that is the same in all lanes, summed in scalar registers.  (Left to itself the compiler adds the lane's offset to the array's
// address outside the loop, and keeps a pair of vector registers for every array.)
typedef __attribute__((address_space(1))) const uint8_t* Base;
__device__ __forceinline__ Base base_of(const void* p, int64_t bytes) {
    uint64_t v = (uint64_t)p + bytes;
    __asm__("" : "+s"(v));
    return (Base)v;
}
template <class T>
__device__ __forceinline__ T load_at(Base base, uint32_t offset) {
    typedef __attribute__((address_space(1))) const T* At;
    return *(At)(base + offset);
}

template <bool BF, int ND>
struct Reader {
    const AttendArgs& A;
    const int32_t* table;      // the sequence's pages
    int h, last_half;          // cache head; start of the last 16 tokens that the table has room for
    int lane, n, q;

    // Page of the 16 tokens from `at`, or of the last ones that the table has room for.  Past the sequence's end its entries may be
    // anything; what is read by them lies in the cache and is not used.
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
    __device__ __forceinline__ void load_keys(Codes<ND>& f, const int64_t (&row)[2]) const {
        const uint32_t of = n * (16 * ND) + q * (4 * ND);
        typedef uint32_t uintx3 __attribute__((ext_vector_type(3)));
        typedef uint32_t uintx4_at4 __attribute__((ext_vector_type(4), aligned(4)));
        typedef uint32_t uintx3_at4 __attribute__((ext_vector_type(3), aligned(4)));
        typedef uint32_t uintx2_at4 __attribute__((ext_vector_type(2), aligned(4)));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const Base base = base_of(A.c.k_codes, row[u] * (16 * ND));
            if constexpr (ND >= 4) {
                const uintx4 v = load_at<uintx4_at4>(base, of);
                f.k[u][0] = v[0]; f.k[u][1] = v[1]; f.k[u][2] = v[2]; f.k[u][3] = v[3];
            }
            constexpr int done = ND & 4 || ND == 8 ? 4 : 0;
            if constexpr (ND == 8) {
                const uintx4 v = load_at<uintx4_at4>(base, of + 16);
                f.k[u][4] = v[0]; f.k[u][5] = v[1]; f.k[u][6] = v[2]; f.k[u][7] = v[3];
            } else if constexpr (ND - done == 3) {
                const uintx3 v = load_at<uintx3_at4>(base, of + 4 * done);
                f.k[u][done] = v[0]; f.k[u][done + 1] = v[1]; f.k[u][done + 2] = v[2];
            } else if constexpr (ND - done == 2) {
                const uintx2 v = load_at<uintx2_at4>(base, of + 4 * done);
                f.k[u][done] = v[0]; f.k[u][done + 1] = v[1];
            } else if constexpr (ND - done == 1) {
                f.k[u][done] = load_at<uint32_t>(base, of + 4 * done);
            }
        }
    }
    __device__ __forceinline__ void load_scales(Codes<ND>& f, const int64_t (&row)[2]) const {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f.ks[u] = load_at<uintx2>(base_of(A.c.k_scale, row[u] * 2), 8 * q);
            f.vs[u] = load_at<uintx2>(base_of(A.c.v_scale, row[u] * 2), 8 * q);
        }
    }
    __device__ __forceinline__ void load_values(Codes<ND>& f, const int64_t (&row)[2]) const {
        using P = Pieces<ND>;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const Base base = base_of(A.c.v_codes, row[u] * (16 * ND));
#pragma unroll
            for (int p = 0; p < P::count; ++p) {
                const uint32_t of = q * 4 * (16 * ND) + n * P::width(p);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int more = r * (16 * ND) + 16 * P::before(p);
                    f.v[u][r][p] = P::width(p) == 4 ? load_at<uint32_t>(base, of + more)
                                 : P::width(p) == 2 ? load_at<uint16_t>(base, of + more) : load_at<uint8_t>(base, of + more);
                }
            }
        }
    }
};

template <bool BF>
__device__ __forceinline__ float scale_at(uintx2 s, int r) { return lp_to_float((uint16_t)(s[r / 2] >> 16 * (r & 1)), BF); }

// The table of pairs of levels in LDS: 256 rows of 32 pairs of the keys' levels and 32 of the values'.
struct Table {
    static constexpr int bytes = 65536;

    // the pair of byte b of the word; copy = 4 (lane % 32)
    template <bool VALUES>
    static __device__ __forceinline__ uint32_t pair(const uint8_t* lds, uint32_t word, int b, uint32_t copy) {
        return *(const uint32_t*)(lds + __builtin_amdgcn_perm(word, copy, 0x0c0c0400u | (uint32_t)b << 8) + (VALUES ? 128 : 0));
    }

    // The level that a lane brings to `fill`: lanes 0..15 the keys', lanes 16..31 the values'.
    static __device__ __forceinline__ uint16_t level(const KVView& c, int h, int lane) {
        return ((lane & 16) ? c.v_levels : c.k_levels)[h * 16 + (lane & 15)];
    }
    // A row is sixteen pieces of 16 bytes, eight of the keys and eight of the values.  -> what products with the values' levels come times
    template <bool BF, int THREADS>
    static __device__ __forceinline__ float fill(uint8_t* lds, uint16_t level, int lane) {
        float down = 1.f;
        uint32_t mine = level;
        if constexpr (BF) {
            int top = level & 0x7fff;                             // the largest of 16 lanes: rotated by 8, 4, 2 and 1 (the table waits for it)
            top = max(top, __builtin_amdgcn_mov_dpp(top, 0x128, 0xf, 0xf, false));
            top = max(top, __builtin_amdgcn_mov_dpp(top, 0x124, 0xf, 0xf, false));
            top = max(top, __builtin_amdgcn_mov_dpp(top, 0x122, 0xf, 0xf, false));
            top = max(top, __builtin_amdgcn_mov_dpp(top, 0x121, 0xf, 0xf, false));
            // biased exponents: 2^(14 - e) has 127 + 14 - (E - 127)
            const int up = min(268 - (__builtin_amdgcn_readlane(top, 16) >> 7), 253);
            down = __uint_as_float((uint32_t)(254 - up) << 23);
            if (lane & 16) mine = float_to_half(lp_to_float(level, true) * __uint_as_float((uint32_t)up << 23));
        }
        const int side = lane & 8 ? 16 : 0;
#pragma unroll 2
        for (int i = 0; i < bytes / 16 / THREADS; ++i) {
            const int at = i * THREADS + threadIdx.x, code = at / 16;
            const uint32_t pair = (uint32_t)__shfl((int)mine, side + (code & 15)) | ((uint32_t)__shfl((int)mine, side + (code >> 4)) << 16);
            ((uintx4*)lds)[at] = uintx4{pair, pair, pair, pair};
        }
        return down;
    }
};

// Where a sequence's queries are and what they see.
struct Place {
    int len, q0, nq, rows;
    __device__ __forceinline__ Place(const KVAttend& a, const KVView& c, int group, int b) {
        len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
        q0 = a.q_start ? min(max(a.q_start[b], 0), (int)a.Tq) : b * a.max_q;
        nq = a.q_start ? min(min(max(a.q_start[b + 1] - q0, 0), a.max_q), (int)a.Tq - q0) : a.max_q;
        rows = nq * group;
    }
};

// The tokens that a wave's rows see: all of [lo, hi) is seen by some row; the row of column c, at position pos[c], sees those of
// [0, hi) that are more than `before` and at most `after` from it.
template <int NT>
struct Seen {
    int lo, hi, before, after, pos[NT];
};

// Query rows from row0 on: the operand, and where the columns' rows are.
template <int ND, int NT>
__device__ __forceinline__ void load_queries(const AttendArgs& A, const Place& p, int h, int row0, int n, int q, uintx4 (&Q)[NT][ND],
                                             Seen<NT>& seen) {
    const KVAttend& a = A.a;
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const int row = row0 + c * 16 + n, i = A.group.quotient(row), g = row - i * A.group.by;
        const bool live = row < p.rows;
        const uint16_t* at = a.q.at + (int64_t)(p.q0 + i) * a.q.token + (int64_t)(h * A.group.by + g) * a.q.head + q * (8 * ND);
#pragma unroll
        for (int k = 0; k < ND; ++k) {
            Q[c][k] = uintx4{0, 0, 0, 0};
            if (live) Q[c][k] = *(const uintx4_any*)(at + 8 * k) ^ A.flip;
        }
        seen.pos[c] = p.len - p.nq + i;
    }
    seen.after = a.causal ? 0 : INT32_MAX;
    seen.before = a.window ? -a.window : INT32_MIN;
}

// 1 / sum, 0 for a row that has seen nothing; and its lse (top in powers of two)
__device__ __forceinline__ float inverse(float sum) { return sum > 0.f || sum != sum ? 1.f / sum : 0.f; }
__device__ __forceinline__ float lse_of(float top, float sum) {
    return sum > 0.f || sum != sum ? (top + __log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

// References and sums of a wave's rows; a lane keeps its column's, its own tokens' share of the sum.
template <int NT, int S>
struct Softmax {
    float top[NT], sum[NT];    // reference of the exponents (0 before anything is seen), sum of the exponentials
    float bar[NT];             // a score this much above the reference moves it: any before the first, then kMost

    __device__ __forceinline__ Softmax() {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            top[c] = sum[c] = 0.f;
            bar[c] = kNone;
        }
    }

    // One step's scores X (before the keys' scales ks, which come times scale log2 e) become weights w; products O move with their
    // reference.  The lane's e-th score is of token first + 16 (e / 4) + e % 4, vs has its values' scales, 16 bits
    // each, and loses those that must not be multiplied.  A column's reference depends on what its row sees and on nothing else: other columns'
    // scores and scales that the row does not see may bring the wave to the branch, but do not move it there.
    template <bool BF>
    __device__ __forceinline__ void step(const floatx4 (&X)[2][NT], const float (&ks)[8], uintx2 (&vs)[2], bool masked,
                                         const Seen<NT>& seen, int first, floatx4 (&O)[S][NT], uintx4 (&w)[NT]) {
        float x[NT][8], peak[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] = fmaf(X[e / 4][c][e & 3], ks[e], -top[c]);
        // The largest of the lane's scales, as 16-bit integers
        auto largest = [&] {
            const uint32_t two = pk_max_u16(pk_max_u16(vs[0][0], vs[0][1]), pk_max_u16(vs[1][0], vs[1][1]));
            return (uint16_t)max(two & 0xffffu, two >> 16);
        };
        uint16_t most = largest();
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int token = first + 16 * (e / 4) + (e & 3);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    x[c][e] = token >= seen.hi || token - seen.pos[c] > seen.after || token - seen.pos[c] <= seen.before ? -INFINITY : x[c][e];
            }
            // A value's scale that is not finite goes straight to the sums of the rows that see it, and is not multiplied where none does; past the
            // end it may be anything, signs included.
            constexpr uint16_t finite = BF ? 0x7f7f : 0x7bff;
            if (__any(most > finite)) {
                uint32_t bad_for = 0;                             // columns of the lane
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int token = first + 16 * (e / 4) + (e & 3);
                    const bool bad = (vs[e / 4][(e & 3) / 2] >> 16 * (e & 1) & 0x7fffu) > finite, out = bad || token < seen.lo || token >= seen.hi;
#pragma unroll
                    for (int c = 0; c < NT; ++c) bad_for |= bad && !(x[c][e] == -INFINITY) ? 1u << c : 0u;
                    vs[e / 4][(e & 3) / 2] &= out ? (e & 1 ? 0x0000ffffu : 0xffff0000u) : 0xffffffffu;
                }
                most = largest();
                bad_for |= __shfl_xor((int)bad_for, 16);
                bad_for |= __shfl_xor((int)bad_for, 32);
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int s = 0; s < S; ++s) O[s][c] += bad_for >> c & 1 ? NAN : 0.f;
            }
        }
        // Scales are positive and order as integers, the largest is below a power of two: scores below `fits` give weights that fit
        const float fits = kFits - (float)__builtin_amdgcn_frexp_expf(lp_to_float(most, BF));
        bool move = false;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            peak[c] = x[c][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) peak[c] = fmaxf(peak[c], x[c][e]);
            move |= peak[c] > fminf(bar[c], fits);
        }
        if (__any(move)) {
            uintx2 rare[2] = {vs[0], vs[1]};                      // (scales converted here are not to be kept in registers for below)
            __asm__("" : "+v"(rare[0]), "+v"(rare[1]));
            float log_v[8];                                       // (one that is not finite has its part in the products, not in the reference)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = scale_at<BF>(rare[e / 4], e & 3);
                log_v[e] = v <= 3.402823466e38f ? __builtin_amdgcn_logf(v) : -INFINITY;
            }
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                float score = peak[c], weight = kNone;
#pragma unroll
                for (int e = 0; e < 8; ++e) weight = fmaxf(weight, x[c][e] + log_v[e]);
                score = fmaxf(score, __shfl_xor(score, 16));
                score = fmaxf(score, __shfl_xor(score, 32));
                weight = fmaxf(weight, __shfl_xor(weight, 16));
                weight = fmaxf(weight, __shfl_xor(weight, 32));
                // before anything is seen sum and products are zero, and the first reference may lie anywhere
                const bool first = bar[c] == kNone;
                const bool moves = score > bar[c] || (!first && weight > kFits + 0.01f);   // (a rounding above what brings a lane here)
                const float by = moves ? fmaxf(weight - kTop, score - kMostMoved) : 0.f;
                bar[c] = moves ? kMost : bar[c];
                top[c] += by;
                sum[c] = first ? 0.f : times_exp2(sum[c], -by);
                const float shrink = first ? 0.f : exp2_fast(-by);
#pragma unroll
                for (int s = 0; s < S; ++s) O[s][c] *= shrink;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] -= by;
            }
        }
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = scale_at<BF>(vs[e / 4], e & 3);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[c][e] = exp2_fast(x[c][e]);
                sum[c] += x[c][e];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) w[c][j] = pack_products(x[c][2 * j], v[2 * j], x[c][2 * j + 1], v[2 * j + 1]);
        }
    }

    // The columns' sums, and products with the values' levels as they are
    __device__ __forceinline__ void finish(floatx4 (&O)[S][NT], float down) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            sum[c] += __shfl_xor(sum[c], 16);
            sum[c] += __shfl_xor(sum[c], 32);
#pragma unroll
            for (int s = 0; s < S; ++s) O[s][c] *= down;
        }
    }
};

// JOIN: the waves of a workgroup share the rows and divide the tokens, each takes every kJoinWaves-th step (and workgroups may divide them
// further); otherwise each wave has rows of its own, of one sequence or, where that has fewer tiles than a workgroup has waves, of
// several, and takes all steps that they see.  Codes go straight from the cache into operands.
template <bool BF, int ND, int NT, bool JOIN>
__global__ __launch_bounds__(64 * (JOIN ? kJoinWaves : own_waves(NT)), NT == 1 && ND <= 4 ? 4 : JOIN ? 1 : 2)
void kv_attend_kernel(AttendArgs A) {
    // (a fixed size, so that the compiler knows the table's address and leaves it to the instruction's offset)
    using T = Table;
    __shared__ __align__(16) uint8_t lds[T::bytes + (JOIN ? 2 * kJoinWaves * 16 * NT * 4 : 0)];
    using P = Pieces<ND>;
    constexpr int R = 16 * NT, S = 2 * ND, W = JOIN ? kJoinWaves : 1, WAVES = JOIN ? kJoinWaves : own_waves(NT), THREADS = 64 * WAVES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    // row_blocks: of a sequence, workgroups where its waves share the rows, tiles otherwise
    int h, b, split = 0, rb;
    bool some = true;                                             // whether there is such a sequence
    const bool packed = !JOIN && A.row_blocks < WAVES;
    if constexpr (JOIN) {
        h = blockIdx.y, b = blockIdx.z, split = blockIdx.x % A.splits, rb = blockIdx.x / A.splits;
    } else {
        h = blockIdx.x % A.c.heads;
        const int block = blockIdx.x / A.c.heads;
        if (packed) {
            const int unit = block * WAVES + wave, sequence = unit / A.row_blocks;
            some = sequence < A.a.B;
            b = min(sequence, A.a.B - 1), rb = unit - sequence * A.row_blocks;
        } else {                                                  // the tiles with the most tokens first
            b = block % A.a.B, rb = ((A.row_blocks - 1) / WAVES - block / A.a.B) * WAVES + wave;
        }
    }
    const KVAttend& a = A.a;
    const uint16_t level = T::level(A.c, h, lane);                // (the first load: the table waits for it alone)

    // Without a window the first step does not depend on the sequence's length, and its loads are issued before that is known.
    Reader<BF, ND> in{A, a.pages + (int64_t)b * a.max_pages, h, (a.max_pages << A.c.page_shift) - 16, lane, n, q};
    int ahead = 0, mine = JOIN ? split * A.chunk + wave * kStep : 0;   // lane l: page of half l % 2 of step l / 2 of this batch; first step
    auto pages_from = [&](int step) { return in.page_of(mine + (step + lane / 2) * W * kStep + (lane & 1) * 16); };
    Codes<ND> f;                                                  // the step's, refilled piece by piece as it is used up
    int64_t row[2];
    auto begin = [&] {
        ahead = pages_from(0);
        in.rows_of(row, mine, __builtin_amdgcn_readlane(ahead, 0), __builtin_amdgcn_readlane(ahead, 1));
        in.load_keys(f, row);
        in.load_scales(f, row);
        in.load_values(f, row);
    };
    if (!a.window) begin();

    const Place at(a, A.c, A.group.by, b);
    const int rows = some ? at.rows : 0, len = at.len, q0 = at.q0, nq = at.nq, row0 = rb * R;
    if (JOIN ? row0 >= rows : !packed && (rb - wave) * R >= rows) return;   // the whole workgroup

    // tokens that the wave's rows see
    const int i0 = A.group.quotient(row0), i1 = A.group.quotient(max(min(row0 + R, rows) - 1, 0));
    const int p0 = len - nq + i0, p1 = len - nq + i1;
    const int hi = row0 >= rows ? 0 : a.causal ? max(min(len, p1 + 1), 0) : len;
    const int lo = a.window ? max(0, p0 - a.window + 1) : 0;
    const int first = (lo & ~(kStep - 1)) + (JOIN ? split * A.chunk : 0);
    const int end = !JOIN || split == A.splits - 1 ? hi : min(hi, first + A.chunk);
    if (JOIN && split > 0 && first >= hi) return;                 // the whole workgroup
    // a step is whole where every row sees all of its tokens
    const int whole_end = a.causal ? min(len, p0 + 1) : len, whole_from = a.window ? p1 - a.window + 1 : 0;
    mine = first + (JOIN ? wave * kStep : 0);
    const int steps = end > mine ? (end - mine + W * kStep - 1) / (W * kStep) : 0;
    if (a.window && steps) begin();

    uintx4 Q[NT][ND];
    Seen<NT> seen;
    seen.lo = lo;
    seen.hi = hi;
    load_queries<ND, NT>(A, at, h, row0, n, q, Q, seen);
    const float down = T::fill<BF, THREADS>(lds, level, lane);

    floatx4 O[S][NT];
    Softmax<NT, S> soft;
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int s = 0; s < S; ++s) O[s][c] = floatx4{0, 0, 0, 0};
    const uint32_t copy = (lane & 31) * 4;
    __syncthreads();

    for (int it = 0; it < steps; ++it) {
        const int from = mine + it * W * kStep;
        if ((it + 1) % kPagesAhead == 0) ahead = pages_from(it + 1);
        const int l = 2 * ((it + 1) % kPagesAhead);
        // rows of the next step (after the last one: of the sequence's end, not used)
        in.rows_of(row, from + W * kStep, __builtin_amdgcn_readlane(ahead, l), __builtin_amdgcn_readlane(ahead, l + 1));

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
                for (int j = 0; j < 4; ++j) op[j] = T::pair<false>(lds, f.k[u][k], j, copy);
#pragma unroll
                for (int c = 0; c < NT; ++c) X[u][c] = mfma16<BF>(op, Q[c][k], X[u][c]);
            }
        if constexpr (!JOIN) __builtin_amdgcn_sched_barrier(0);
        in.load_keys(f, row);

        float ks[8];
        uintx2 vs[2] = {f.vs[0], f.vs[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) ks[e] = scale_at<BF>(f.ks[e / 4], e & 3) * A.scale_log2;
        in.load_scales(f, row);
        if constexpr (!JOIN) __builtin_amdgcn_sched_barrier(0);
        uintx4 w[NT];
        soft.template step<BF>(X, ks, vs, from + kStep > whole_end || from < whole_from,   // some row does not see all of these tokens
                               seen, from + 4 * q, O, w);

        if constexpr (!JOIN) __builtin_amdgcn_sched_barrier(0);
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
                    for (int j = 0; j < 4; ++j) op[j] = T::pair<true>(lds, pairs[j][half], i, copy);
                    const int s = 2 * (P::before(p) + i) + half;
#pragma unroll
                    for (int c = 0; c < NT; ++c) O[s][c] = mfma16<false>(op, w[c], O[s][c]);
                }
        }
        if constexpr (!JOIN) __builtin_amdgcn_sched_barrier(0);
        in.load_values(f, row);
    }

    soft.finish(O, down);
    float (&top)[NT] = soft.top, (&sum)[NT] = soft.sum;

    int last0 = row0;
    __asm__("" : "+s"(last0));                                    // (places of the result are found now, not kept in registers all along)
    if constexpr (!JOIN) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const int row = last0 + c * 16 + n, i = A.group.quotient(row), g = row - i * A.group.by;
            if (row >= rows) continue;
            const int64_t to = (int64_t)(q0 + i) * a.q_heads + h * A.group.by + g;
            const float inv = inverse(soft.sum[c]);
            // a piece's channels of one of O^T's rows lie side by side
#pragma unroll
            for (int p = 0; p < P::count; ++p)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t o[P::width(0)];
#pragma unroll
                    for (int j = 0; j < P::width(p); ++j) {
                        const int s = 2 * (P::before(p) + j);
                        o[j] = float_to_lp_any(O[s][c][r] * inv, BF) | (uint32_t)float_to_lp_any(O[s + 1][c][r] * inv, BF) << 16;
                    }
                    uint16_t* out = a.out + to * (32 * ND) + 2 * (16 * P::before(p) + (4 * q + r) * P::width(p));
                    if constexpr (P::width(0) == 4)
                        if (P::width(p) == 4) *(uintx4*)out = uintx4{o[0], o[1], o[2], o[3]};
                    if constexpr (P::width(0) >= 2)
                        if (P::width(p) == 2) *(uintx2*)out = uintx2{o[0], o[1]};
                    if (P::width(p) == 1) *(uint32_t*)out = o[0];
                }
            if (a.lse && q == 0) a.lse[to] = lse_of(soft.top[c], soft.sum[c]);
        }
        return;
    }

    const bool partial = A.splits > 1 && (hi - (lo & ~(kStep - 1))) > A.chunk;
    float* part = a.part + ((((int64_t)b * A.c.heads + h) * A.row_blocks + rb) * A.splits + split) * (R * (32 * ND + 2));
    auto finish = [&](int c, int s, floatx4 o, float t, float l) {
        const int row = last0 + c * 16 + n, i = A.group.quotient(row), g = row - i * A.group.by;
        if (row >= rows) return;
        const int64_t at = (int64_t)(q0 + i) * a.q_heads + h * A.group.by + g;
        const float inv = inverse(l);
#pragma unroll
        for (int r = 0; r < 4; ++r) a.out[at * (32 * ND) + channel_of<ND>(s, 4 * q + r)] = float_to_lp_any(o[r] * inv, BF);
        if (a.lse && s == 0 && q == 0) a.lse[at] = lse_of(t, l);
    };

    if constexpr (JOIN) {
        // The waves' maxima and sums, then their products by way of the table's memory, a few subtiles at a time.
        static_assert(kJoinWaves == 8, "eight of them, two pieces of 16 bytes");
        floatx4* tops = (floatx4*)(lds + T::bytes);               // [R][waves]
        floatx4* sums = tops + R * 2;
        if (q == 0)
#pragma unroll
            for (int c = 0; c < NT; ++c) ((float*)(tops + (c * 16 + n) * 2))[wave] = sum[c] == 0.f ? kNone : top[c];
        __syncthreads();                                          // the table is done with, too
        float t[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const floatx4 u = tops[(c * 16 + n) * 2], v = tops[(c * 16 + n) * 2 + 1];
            t[c] = fmaxf(fmaxf(fmaxf(u[0], u[1]), fmaxf(u[2], u[3])), fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
            const float mine = sum[c] == 0.f ? 0.f : exp2_fast(top[c] - t[c]);
            if (q == 0) ((float*)(sums + (c * 16 + n) * 2))[wave] = sum[c] == 0.f ? 0.f : times_exp2(sum[c], top[c] - t[c]);
#pragma unroll
            for (int s = 0; s < S; ++s) O[s][c] *= mine;
        }
        constexpr int AT_ONCE = (int)(T::bytes / 16) / (64 * kJoinWaves * NT);
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
                const floatx4 l4 = sums[(c * 16 + n) * 2] + sums[(c * 16 + n) * 2 + 1];
                const float lc = (l4[0] + l4[1]) + (l4[2] + l4[3]);
                float tc = t[0];
#pragma unroll
                for (int j = 1; j < NT; ++j) tc = c == j ? t[j] : tc;
                if (partial) {
                    if (last0 + c * 16 + n >= rows) continue;
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

// Joins the splits of one subtile of one row block.  All their maxima and sums are read at once, 16 columns by 4 splits a wave, and become
// the splits' factors in LDS; then each of the waves adds its share of the splits' products, and the first wave what they have.  Few
// splits (many sequences) take one wave, many eight.  What the workspace holds is read before it is known which splits have written
// anything; the others are left out afterwards, whatever their places hold.
template <bool BF, int ND, int NT, int WAVES, int MOST>
__global__ __launch_bounds__(64 * WAVES, 4) void kv_join_kernel(AttendArgs A) {
    constexpr int R = 16 * NT, LANES = 4 * WAVES, EACH = MOST / LANES, EARLY = 4;
    __shared__ floatx4 swap[WAVES][64];
    __shared__ float factor[MOST][16], most[WAVES][16], all[WAVES][16];
    const KVAttend& a = A.a;
    const int b = blockIdx.z, h = blockIdx.y, tile = blockIdx.x % (2 * ND * NT), rb = blockIdx.x / (2 * ND * NT);
    const int s = tile / NT, c = tile % NT;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int64_t stride = R * (32 * ND + 2);
    const float* part = a.part + (((int64_t)b * A.c.heads + h) * A.row_blocks + rb) * A.splits * stride;
    const float* products = part + 2 * R + ((s * NT + c) * 64 + lane) * 4;
    const int col = c * 16 + n;

    float tops[EACH], sums[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int i = k * LANES + wave * 4 + q;
        tops[k] = i < A.splits ? part[i * stride + col] : kNone;
        sums[k] = i < A.splits ? part[i * stride + R + col] : 0.f;
    }
    floatx4 early[EARLY];
#pragma unroll
    for (int k = 0; k < EARLY; ++k) early[k] = *(const floatx4*)(products + min(k * WAVES + wave, A.splits - 1) * stride);

    const Place place(a, A.c, A.group.by, b);
    const int rows = place.rows, len = place.len, q0 = place.q0, nq = place.nq, row0 = rb * R;
    if (row0 + c * 16 >= rows) return;
    const int i0 = A.group.quotient(row0), i1 = A.group.quotient(min(row0 + R, rows) - 1);
    const int hi = a.causal ? max(min(len, len - nq + i1 + 1), 0) : len;
    const int lo = (a.window ? max(0, len - nq + i0 - a.window + 1) : 0) & ~(kStep - 1);
    if (hi - lo <= A.chunk) return;                               // one split has written the result itself
    const int parts = min(A.splits, (hi - lo + A.chunk - 1) / A.chunk);

    float t = kNone, l = 0.f;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const bool has = k * LANES + wave * 4 + q < parts;
        tops[k] = has ? tops[k] : kNone;
        sums[k] = has ? sums[k] : 0.f;
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
        factor[k * LANES + wave * 4 + q][n] = exp2_fast(tops[k] - t);
        l += times_exp2(sums[k], tops[k] - t);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (q == 0) all[wave][n] = l;
    __syncthreads();

    floatx4 o = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < EARLY; ++k) {
        const int i = k * WAVES + wave;
        if (i < parts) o += factor[i][n] * early[k];
    }
#pragma unroll 2
    for (int i = EARLY * WAVES + wave; i < parts; i += WAVES) o += factor[i][n] * *(const floatx4*)(products + i * stride);
    swap[wave][lane] = o;
    __syncthreads();
    const int row = row0 + col;
    if (wave || row >= rows) return;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) l += all[w][n];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) o += swap[w][lane];
    const int i = A.group.quotient(row), g = row - i * A.group.by;
    const int64_t at = (int64_t)(q0 + i) * a.q_heads + h * A.group.by + g;
    const float inv = inverse(l);
#pragma unroll
    for (int r = 0; r < 4; ++r) a.out[at * (32 * ND) + channel_of<ND>(s, 4 * q + r)] = float_to_lp_any(o[r] * inv, BF);
    if (a.lse && s == 0 && q == 0) a.lse[at] = lse_of(t, l);
}

// Most tiles of a wave: as many as leave room for two waves a SIMD without spills (O takes 8 registers a tile and 32 channels, q 4).  With
// one more, 2 sequences of 1024 queries over 4096 tokens, 16 query heads: d = 256 two tiles 462 us, one 246; d = 224 337 and 238.  With
// one less: d = 128 chunk as above two tiles 1176 us, three 1054.
static constexpr int own_tiles(int ND) { return ND <= 2 ? 4 : ND <= 4 ? 3 : ND <= 6 ? 2 : 1; }
static constexpr int join_tiles(int ND) { return ND <= 2 ? 4 : ND <= 4 ? 3 : ND <= 6 ? 2 : 1; }

KVPlan choose_kv_plan(const KVView& c, int q_heads, int B, int max_q, int64_t reach) {
    const int group = q_heads / c.heads, ND = c.d / 32;
    const int64_t rows = (int64_t)max_q * group, units = device_cu_count();
    KVPlan p;
    p.splits = 1;
    p.chunk = INT32_MAX / 2;
    // Waves with rows of their own need no exchange at the end, but the rows' workgroups alone have to fill the chip (8 x 5 queries of 16
    // heads of 256 over 4000 tokens: 16 workgroups 235 us, divided by tokens too 23); otherwise the tokens are divided.
    const int64_t own_blocks = (int64_t)B * c.heads * cdiv(rows, 16 * own_tiles(ND) * own_waves(own_tiles(ND)));
    if (rows > 16 * join_tiles(ND) && own_blocks >= units) {
        p.join = false;
        p.tiles = own_tiles(ND);
        p.row_blocks = (int)cdiv(rows, 16 * p.tiles);
        return p;
    }
    p.join = true;
    p.tiles = (int)std::min(cdiv(rows, 16), (int64_t)join_tiles(ND));
    p.row_blocks = (int)cdiv(rows, 16 * p.tiles);
    // One workgroup to a compute unit: 8 heads, one sequence of 131072 tokens 64 splits 38.2 us, 32 35.6, 24 41.4.
    const int64_t wg = kJoinWaves * kStep, blocks = (int64_t)B * c.heads * p.row_blocks;
    const int64_t want = blocks >= units ? 1 : units / blocks, steps = cdiv(reach, wg);
    // Splitting costs the second launch, about four steps of a workgroup: 8 heads of 128, one sequence of 700 tokens (3 steps) 10.1 us
    // in one piece and 10.0 in three, of 1500 (6) 13.8 and 10.4 in six; 24 sequences of 2048 (8), 4 heads of 64, 13.3 and 13.0 in two.
    p.splits = (int)std::min({want, steps, (int64_t)kMostSplits});
    if (steps - cdiv(steps, p.splits) <= 4) p.splits = 1;
    if (p.splits > 1) {
        p.chunk = cdiv(steps, p.splits) * wg;
        return p;
    }
    // Many short sequences: a tile to a wave, eight to a workgroup, saves the workgroups' fixed cost and gives up dividing the tokens.  In tenths of a
    // microsecond, fitted to 986 measured pairs from 32 to 256 channels, 1 to 4 tiles and 9 to 500 tokens (of which it takes the slower one where that
    // costs 0.6 % on average, and tiles where they are up to 2 % slower): workgroups that share their rows and hold at most 128 registers run in
    // pairs on a compute unit, others in rounds; each takes a time of its own and one a step of 256 tokens.  Tiles take theirs a step of 32.
    // One query of 4 heads to each of 8 heads of 128: 64 sequences of 100 tokens 10.3 us shared and 10.7 in tiles, of 32 9.5 and 6.6; 128 of 300
    // 23 and 18; of 256 channels 64 of 200 22.6 and 21.5, 32 of 200 12.4 and 21.2.
    const int64_t tiles = cdiv(rows, 16), own = cdiv(B * tiles, 8) * c.heads, more = std::max(blocks - units, (int64_t)0),
                  more_own = std::max(own - units, (int64_t)0), w = ND * p.tiles, own_steps = cdiv(reach, kStep);
    const bool pairs = w <= 2 || (p.tiles == 1 && ND <= 4);
    const int64_t shared_cost = pairs ? (40 + 5 * w + (4 + 3 * w) * steps) * units + (15 + w + (7 + 2 * w) * steps) * more
                                      : (60 + 2 * w + (10 + 2 * w) * steps) * cdiv(blocks, units) * units;
    const int64_t own_cost = (38 + 4 * ND + (7 + 2 * ND) * own_steps) * units + (15 + 9 * ND + (6 + 6 * ND) * own_steps) * more_own;
    if (own_cost < shared_cost) {
        p.join = false;
        p.tiles = 1;
        p.row_blocks = (int)tiles;
    }
    return p;
}

template <bool BF, int ND, int NT>
static fk_status launch_form(const AttendArgs& A, hipStream_t s) {
    kv_attend_kernel<BF, ND, NT, true><<<dim3(A.row_blocks * A.splits, A.c.heads, A.a.B), 64 * kJoinWaves, 0, s>>>(A);
    FK_HIP(hipGetLastError());
    if (A.splits > 1) {
        const dim3 grid(A.row_blocks * 2 * ND * NT, A.c.heads, A.a.B);
        if (A.splits <= 8) kv_join_kernel<BF, ND, NT, 1, 8><<<grid, 64, 0, s>>>(A);
        else kv_join_kernel<BF, ND, NT, 8, kMostSplits><<<grid, 512, 0, s>>>(A);
        FK_HIP(hipGetLastError());
    }
    return FK_OK;
}

template <bool BF, int ND>
static fk_status launch_width(const AttendArgs& A, const KVPlan& p, hipStream_t s) {
    if (!p.join) {
        const int waves = own_waves(p.tiles);
        const int64_t blocks = (A.row_blocks < waves ? cdiv((int64_t)A.a.B * A.row_blocks, waves) : cdiv(A.row_blocks, waves) * A.a.B) * A.c.heads;
        if (blocks > INT32_MAX / 512) {
            set_error("fk_kv_attend: unsupported size: %lld workgroups", (long long)blocks);
            return FK_EUNSUPPORTED;
        }
        if (p.tiles == 1) kv_attend_kernel<BF, ND, 1, false><<<(unsigned)blocks, 64 * own_waves(1), 0, s>>>(A);
        else if constexpr (own_tiles(ND) > 1)
            kv_attend_kernel<BF, ND, own_tiles(ND), false><<<(unsigned)blocks, 64 * own_waves(own_tiles(ND)), 0, s>>>(A);
        FK_HIP(hipGetLastError());
        return FK_OK;
    }
    if (p.tiles == 1) return launch_form<BF, ND, 1>(A, s);
    if constexpr (join_tiles(ND) >= 2)
        if (p.tiles == 2) return launch_form<BF, ND, 2>(A, s);
    if constexpr (join_tiles(ND) >= 3)
        if (p.tiles == 3) return launch_form<BF, ND, 3>(A, s);
    return launch_form<BF, ND, join_tiles(ND)>(A, s);
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
    const AttendArgs A{c, a, Divider(a.q_heads / c.heads), p.splits, p.row_blocks, (int)p.chunk, fmaxf(fabsf(a.scale) * 1.44269504088896341f, 1e-37f), a.scale < 0.f ? 0x80008000u : 0u};
    return c.bf ? launch_type<true>(A, p, s) : launch_type<false>(A, p, s);
}

}  // namespace fk
