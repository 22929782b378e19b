// Attention weights of cached tokens, added up over queries.
//
// w_t = (t known ? decay w_t : 0) + sum over query rows n that see t of 2^(scale log2 e s_t (q_n . K_t) - log2 e lse_n), a row being one head of
// the group at one query token, s_t the key's scale, lse_n the logarithm of the row's softmax sum, which attention has left.  No maximum is
// searched: the logarithm brings the weights to at most 1.
//
// A wave takes 64 tokens (32 of wide rows where queries stream by): S = q K^T by 16x16x32 MFMA with 16 query rows and 16 tokens, so that a lane
// owns one token of 4 rows and adds up its weights in registers.  Keys become operands as in attention, by a table of pairs of levels in LDS, once
// for all rows.  Queries lie in LDS in the order in which the lanes read them.  The four quarters of a wave are added at the end by two
// exchanges, which leave token l in lane l.  A token belongs to one workgroup, or, where rows are divided among several, a second kernel
// adds their parts in order: no atomics, and no result depends on the order of workgroups.
//
// Two forms.  Few rows (up to 128 at 128 channels) stay in LDS, and waves go over the tokens with the next step's codes on their way; the
// workgroup's four waves a SIMD hide the rest.  Bound by bytes: 64 sequences of up to 8192 tokens, 8 heads of 128, 198 MB in 52 us, 3.8 TB/s
// (one of 700: 4.8 us).  A tile's read, products and exponentials follow each other there, so that with some dozen rows they bound it instead: 6 x 32
// queries of 64 channels over up to 15000 tokens 17 us, where bytes take 4.  More rows stream by in blocks of two buffers, rows that all see all tokens with the products of a tile under
// the exponentials of the one before it: 2 x 4096 queries of 32 heads over up to 9000 tokens, 426 GFLOP in 481 us, 0.89 PFLOP/s
// (256 channels: three registers go through scratch memory).
// A tile of 16 rows and 64 tokens at d = 128 is 16 MFMA (256 cycles) and 16 times multiply-add, exponential and addition (another 256); alone
// in a loop the two overlap to 412, here they take about 500: the rest is what a wave needs between tiles and at the blocks' barriers.
// (The simple form, tokens on the tiles' row side and each wave reading the queries from memory: 1019 us.  Keys of 32 tokens and four waves a SIMD spill:
// 1054.  16-byte pieces gathered in the lanes' order instead of whole rows: 774 against 609 at that step.)
#include <algorithm>
#include <type_traits>

#include "fk_device.h"
#include "fk_evict.h"
#include "fk_kv_attend.h"

namespace fk {

constexpr int kWeighWaves = 8, kWeighThreads = 64 * kWeighWaves;

// Rows of queries in one of the two buffers, whole tiles; both together are all that a workgroup keeps.
// Where queries stream by, blocks are larger, so that fewer barriers wait for the slowest wave.
constexpr int block_rows(int ND, bool stream) { return (stream ? 512 : 256) / ND / 32 * 32; }
// Tokens of a wave.  Where queries stream by, the keys of all of them are operands meanwhile, and of wide rows registers hold no more.
constexpr int weigh_tokens(int ND, bool stream) { return stream && ND > 4 ? 32 : 64; }

struct WeighArgs {
    KVView c;
    KVWeigh a;
    Divider group;
    int row_waves, blocks, splits;
    int64_t bound;                       // tokens whose rows are divided; whole steps
    int block_rows, block_tokens;        // rows that are put into a buffer at a time; tokens of queries that this is,
    bool whole_tokens;                   // if it is whole ones
    int64_t chunk;
    float scale_log2;
};

// LDS: the table of pairs of the keys' levels, 256 rows of 32 copies, in the lower halves of rows of 256 bytes (a byte of codes is then the
// address with one v_perm), and the queries in the upper ones, in the order in which a wave's lanes read them as operands, 16 bytes a lane.
// Lanes that write a row's pieces meet in a bank unless the rows' order within a piece's slot is turned by the piece, and by no more of the quarter
// than its upper bit, or lanes of two quarters meet when they read (conflicts 39 % of the LDS's time, so 13 %, which the
// cycles do not show: the LDS is busy for a fifth of them).
template <bool STREAM>
struct WeighLds {
    static constexpr int bytes = 65536 * (STREAM ? 2 : 1), piece_bytes = STREAM ? 1024 : 2048;
    static __device__ __forceinline__ int slot_byte(int slot) { return STREAM ? 65536 + slot * 16 : (slot >> 3) * 256 + 128 + (slot & 7) * 16; }
    // piece k of quarter q of row n of a tile
    template <int ND>
    static __device__ __forceinline__ int piece(int tile, int k, int q, int n) {
        return slot_byte((tile * ND + k) * 64 + q * 16 + (n ^ ((q >> 1) * 8) ^ k));
    }
    template <int THREADS>
    static __device__ __forceinline__ void fill(uint8_t* lds, uint16_t level) {
#pragma unroll
        for (int i = 0; i < 256 * 8 / THREADS; ++i) {
            const int at = i * THREADS + threadIdx.x, code = at / 8;
            const uint32_t pair = (uint32_t)__shfl((int)level, code & 15) | ((uint32_t)__shfl((int)level, code >> 4) << 16);
            *(uintx4*)(lds + code * 256 + (at & 7) * 16) = uintx4{pair, pair, pair, pair};
        }
    }
};

// the upper halves of the first and the lower halves of the second register change places, in units of BY lanes
template <int BY>
__device__ __forceinline__ void swap_lanes(float& a, float& b) {
    const auto r = BY == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false)
                            : __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
// Sums of four registers over the four rows of 16 lanes; row u of the result has register u's.
__device__ __forceinline__ float add_rows(float x0, float x1, float x2, float x3) {
    swap_lanes<32>(x0, x2);
    swap_lanes<32>(x1, x3);
    float a = x0 + x2, b = x1 + x3;
    swap_lanes<16>(a, b);
    return a + b;
}

// Order of one tile's products among another's weights: 4 ND products, 16 times two vector instructions and an exponential.
template <int I, int ND>
__device__ __forceinline__ void interleave() {
    if constexpr (I < 16) {
        constexpr int products = (I + 1) * ND / 4 - I * ND / 4;
        if constexpr (products > 0) __builtin_amdgcn_sched_group_barrier(0x8, products, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
        interleave<I + 1, ND>();
    }
}

// STREAM: more query rows than a workgroup keeps; they come by in two buffers, once for every step of tokens.
template <bool BF, int ND, bool STREAM>
__global__ __launch_bounds__(kWeighThreads, !STREAM && ND <= 4 ? 4 : 2) void kv_weigh_kernel(WeighArgs A) {
    constexpr int WAVES = kWeighWaves, THREADS = kWeighThreads, HB = block_rows(ND, STREAM), TILES = HB / 16, EACH = (HB * 4 * ND + THREADS - 1) / THREADS;
    using L = WeighLds<STREAM>;
    // 16 tokens each: of a step, and those whose keys are operands at the same time
    constexpr int TOKENS = weigh_tokens(ND, STREAM), PARTS = TOKENS / 16, HOLD = STREAM ? PARTS : 2;
    __shared__ __align__(16) uint8_t lds[L::bytes];
    __shared__ __align__(16) float logs[2 * HB];                  // of a row: its logarithm in powers of two,
    __shared__ __align__(16) int upto[2 * HB], from[2 * HB];      // and it sees the tokens behind `from` up to `upto`
    __shared__ float parts[WAVES][64];
    constexpr int GROUPS = (HB + 63) / 64;                        // of 64 rows of a buffer: whether one of them
    __shared__ int mute[2][GROUPS];                               // adds nothing, whatever its query and what it sees
    const KVWeigh& a = A.a;
    const KVView& c = A.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    // (the first tokens are seen by the most queries: their workgroups of all sequences and heads come first)
    const int units = c.heads * a.B, unit = blockIdx.x % units, split = blockIdx.x / units % A.splits, block = blockIdx.x / units / A.splits;
    const int h = unit % c.heads, b = unit / c.heads;
    const uint16_t level = c.k_levels[h * 16 + n];
    const int row_waves = STREAM ? 1 : A.row_waves, token_waves = WAVES / row_waves, token_wave = wave & (token_waves - 1), row_wave = wave / token_waves;
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    const int64_t begin64 = block * A.chunk;
    if (begin64 >= len) return;                                   // the whole workgroup
    const int begin = (int)begin64, end = block + 1 == A.blocks ? len : (int)min((int64_t)len, begin64 + A.chunk);
    const int q0 = a.q_start ? min(max(a.q_start[b], 0), (int)a.Tq) : b * a.max_q;
    const int nq = a.q_start ? min(min(max(a.q_start[b + 1] - q0, 0), a.max_q), (int)a.Tq - q0) : a.max_q;
    const int known = a.known ? a.known[b] : len, base = len - nq, rows = nq * A.group.by;
    const int step_tokens = TOKENS * token_waves;
    // Where no query sees any of these tokens, old weights are all there is.  (Where queries stream by, an exit of its own costs scalar registers, and the
    // loops 2.5 %: the steps are gone through without keys and rows.)
    const bool unseen = !nq || (a.window && end - 1 <= base - a.window), idle = STREAM && unseen;
    if (!STREAM && unseen) {
        for (int t = begin + (int)threadIdx.x; t < end; t += THREADS) {
            const int page = a.pages[(int64_t)b * a.max_pages + (t >> c.page_shift)];
            if (page < 0 || page >= c.pages) continue;
            const int64_t at = (((int64_t)page * c.heads + h) << c.page_shift) + (t & ((1 << c.page_shift) - 1));
            a.out[at] = t < known ? a.decay * a.mass[at] : 0.f;
        }
        return;
    }

    // A wave's tokens: page of token t0 + lane, codes, scales and weights so far, one step ahead.
    const int32_t* table = a.pages + (int64_t)b * a.max_pages;
    const int last = (a.max_pages << c.page_shift) - 1;
    int page;
    bool inside;                                                  // whether that page is one of the cache's: otherwise nothing is written
    uint32_t codes[PARTS][ND];
    uint16_t scale = 0;
    float old;
    int64_t at;                                                   // the cache's row of token t0 + lane
    auto ask_page = [&](int t0) { page = table[min(t0 + lane, last) >> c.page_shift]; };
    auto ask = [&](int t0) {
        inside = page >= 0 && page < c.pages;
        page = min(max(page, 0), (int)c.pages - 1);
        at = (((int64_t)page * c.heads + h) << c.page_shift) + (min(t0 + lane, last) & ((1 << c.page_shift) - 1));
        old = inside && t0 + lane < min(known, end) ? a.mass[at] : 0.f;
        if (idle) return;
#pragma unroll
        for (int u = 0; u < PARTS; ++u) {
            const int p = __builtin_amdgcn_readlane(page, 16 * u), first = min(t0 + 16 * u, last - 15) & ((1 << c.page_shift) - 1);
            const Base base = base_of(c.k_codes, ((((int64_t)p * c.heads + h) << c.page_shift) + first) * (16 * ND));
#pragma unroll
            for (int k = 0; k < ND; ++k) codes[u][k] = load_at<uint32_t>(base, n * (16 * ND) + q * (4 * ND) + 4 * k);
        }
        scale = c.k_scale[at];
    };
    ask_page(begin + token_wave * TOKENS);

    // Rows of queries on their way into a buffer, `block_rows` of them: a thread's pieces of 16 bytes, and a row's numbers for the first
    // threads.  As many whole tokens as there is room for, so that from one block to the next a thread's rows only move on by some tokens.
    uintx4 piece[EACH];
    const uint16_t* src[EACH];
    const float* log_at = nullptr;
    float log_in = -INFINITY;
    int pos = 0, upto_in = -1, from_in = INT32_MAX;
#pragma unroll
    for (int e = 0; e < EACH; ++e) piece[e] = uintx4{0, 0, 0, 0};
    auto row_of = [&](int e) { return (e * THREADS + (int)threadIdx.x) / (4 * ND); };
    auto piece_of = [&](int e) { return (e * THREADS + (int)threadIdx.x) % (4 * ND); };
    auto place_rows = [&](int row0) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int row = row0 + row_of(e), i = A.group.quotient(row), g = row - i * A.group.by;
            src[e] = a.q.at + (int64_t)(q0 + i) * a.q.token + (int64_t)(h * A.group.by + g) * a.q.head + piece_of(e) * 8;
        }
        const int row = row0 + threadIdx.x, i = A.group.quotient(row), g = row - i * A.group.by;
        log_at = a.lse + (int64_t)(q0 + i) * a.q_heads + h * A.group.by + g;
        pos = base + i;
    };
    auto ask_rows = [&](int row0, int r_hi) {
        const bool whole = row0 + A.block_rows <= r_hi;
        if (!whole) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) piece[e] = uintx4{0, 0, 0, 0};
        }
        if (HB * 4 * ND == EACH * THREADS && whole && A.block_rows == HB) {   // (no lane is left out)
#pragma unroll
            for (int e = 0; e < EACH; ++e) piece[e] = *(const uintx4_any*)src[e];
        } else {
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (row_of(e) < A.block_rows && (whole || row0 + row_of(e) < r_hi)) piece[e] = *(const uintx4_any*)src[e];
        }
        if (threadIdx.x < HB) {
            const bool live = (int)threadIdx.x < A.block_rows && row0 + (int)threadIdx.x < r_hi;
            log_in = -INFINITY;                                   // (used when it is put down: nothing waits for it here)
            if (live) log_in = *log_at;
            upto_in = !live ? -1 : a.causal ? pos : INT32_MAX;
            from_in = !live ? INT32_MAX : a.window ? pos - a.window : -1;
        }
        if (!A.whole_tokens) return;
#pragma unroll
        for (int e = 0; e < EACH; ++e) src[e] += A.block_tokens * a.q.token;
        log_at += A.block_tokens * a.q_heads;
        pos += A.block_tokens;
    };
    auto put_rows = [&](int buffer) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int row = row_of(e), p = piece_of(e);
            if (row < HB) *(uintx4*)(lds + buffer * (TILES * ND * L::piece_bytes) + L::template piece<ND>(row / 16, p % ND, p / ND, row & 15)) = piece[e];
        }
        if (threadIdx.x < HB) {
            // Of a row that is none, or that has seen nothing: weights of 0.  The second sees nothing here either, and its tiles are masked: its query,
            // or a key that it alone would see, need not be finite.
            const bool none = log_in == -INFINITY;
            logs[buffer * HB + threadIdx.x] = none ? INFINITY : log_in * 1.44269504088896341f;
            upto[buffer * HB + threadIdx.x] = none ? -1 : upto_in;
            from[buffer * HB + threadIdx.x] = from_in;
            const bool any = __any(none && upto_in >= 0);
            if (lane == 0) mute[buffer][wave] = any;
        }
    };
    int tiles = 0;
    if constexpr (!STREAM) {
        tiles = (rows + 15) / 16;
        place_rows(0);
        ask_rows(0, rows);
        put_rows(0);
        if (rows > HB) {
            place_rows(HB);
            ask_rows(HB, rows);
            put_rows(1);
        }
    }
    if (!idle) L::template fill<THREADS>(lds, level);
    ask(begin + token_wave * TOKENS);
    if (!STREAM) __syncthreads();
    auto muted = [&](int buffer) {
        int any = mute[buffer][0];
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) any |= mute[buffer][i];
        return any;
    };
    int hushed = 0;                                               // whether one of the rows that are kept, or of the block, is such a row
    if (!STREAM && tiles) hushed = muted(0) | (rows > HB ? muted(1) : 0);
    const uint32_t copy = (lane & 31) * 4;
    const int q_lane = L::template piece<ND>(0, 0, q, n);           // (piece k: its bits 4 to 6 turned by k)

    for (int step = begin; step < end; step += step_tokens) {
        const int t0 = step + token_wave * TOKENS;
        const bool some = t0 < end, divided = STREAM && A.splits > 1 && step < A.bound;
        if (STREAM && !divided && split) break;                   // (tokens behind the bound that the call names are not divided)
        const int64_t to = inside ? at : -1;
        const float was = old;
        float acc[4] = {0, 0, 0, 0}, ks[4];
        // the scales of tokens 16 u + n
        ks[0] = ks[1] = lp_to_float(scale, BF) * A.scale_log2;
        swap_lanes<16>(ks[0], ks[1]);
        ks[2] = ks[0];
        ks[3] = ks[1];
        swap_lanes<32>(ks[0], ks[2]);
        swap_lanes<32>(ks[1], ks[3]);
        const bool more = t0 + step_tokens < end;
        if (more) ask_page(t0 + step_tokens);

        uintx4 K[HOLD][ND];
        auto decode = [&](int u0) {
#pragma unroll
            for (int u = 0; u < HOLD; ++u)
#pragma unroll
                for (int k = 0; k < ND; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) K[u][k][j] = Table::pair<false>(lds, codes[u0 + u][k], j, copy);
        };
        auto read_tile = [&](int tile, uintx4 (&Q)[ND], floatx4& l) {
#pragma unroll
            for (int k = 0; k < ND; ++k) Q[k] = *(const uintx4*)(lds + (q_lane ^ (k * 16)) + (tile * ND + k) * L::piece_bytes);
            l = *(const floatx4*)(logs + tile * 16 + 4 * q);
        };
        auto scores = [&](const uintx4 (&Q)[ND], floatx4 (&S)[HOLD]) {
#pragma unroll
            for (int u = 0; u < HOLD; ++u) S[u] = floatx4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < ND; ++k)
#pragma unroll
                for (int u = 0; u < HOLD; ++u) S[u] = mfma16<BF>(Q[k], K[u][k], S[u]);
        };
        // the weights of a tile; masked: some of its rows do not see all tokens
        auto add_weights = [&](int tile, const floatx4 (&S)[HOLD], floatx4 l, int u0, bool masked) {
            float w[HOLD][4];
#pragma unroll
            for (int u = 0; u < HOLD; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) w[u][r] = exp2_fast(fmaf(S[u][r], ks[u0 + u], -l[r]));
            if (masked) {
                typedef int intx4 __attribute__((ext_vector_type(4)));
                const intx4 hi = *(const intx4*)(upto + tile * 16 + 4 * q), lo = *(const intx4*)(from + tile * 16 + 4 * q);
#pragma unroll
                for (int u = 0; u < HOLD; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int t = t0 + 16 * (u0 + u) + n;
                        w[u][r] = t <= hi[r] && t > lo[r] ? w[u][r] : 0.f;
                    }
            }
#pragma unroll
            for (int u = 0; u < HOLD; ++u) acc[u0 + u] += (w[u][0] + w[u][1]) + (w[u][2] + w[u][3]);
        };
        auto add_tile = [&](int tile, int u0, bool masked) {
            uintx4 Q[ND];
            floatx4 l, S[HOLD];
            read_tile(tile, Q, l);
            scores(Q, S);
            add_weights(tile, S, l, u0, masked);
        };
        // Where all rows see all tokens, the products of a tile go under the exponentials of the one before it, from block to block.
        constexpr int AHEAD = ND <= 4 ? 2 : 1;                    // tiles of queries in registers (one more does not fit)
        uintx4 Qs[AHEAD][ND];
        floatx4 ls[2], Ss[2][HOLD];
        bool pending = false;                                     // the weights of Ss[1] are to be added yet
        auto flush = [&] {
            if (pending) add_weights(0, Ss[1], ls[1], 0, false);
            pending = false;
        };
        // `count` tiles of rows r0 .. r1 - 1 from place `tile` on, of which this wave takes its share
        auto add_tiles = [&](int tile, int count, int r0, int r1, int u0) {
            const int p0 = base + A.group.quotient(r0), p1 = base + A.group.quotient(r1 - 1), first = t0 + 16 * u0, final = first + 16 * HOLD - 1;
            if ((a.causal && p1 < first) || (a.window && final <= p0 - a.window)) return;   // no row sees any of these tokens
            const bool masked = (a.causal && p0 < final) || (a.window && first <= p1 - a.window) || __builtin_amdgcn_readfirstlane(hushed);
            if (STREAM && !masked && count == TILES) {
                auto place = [&](int i) { return tile + min(i, TILES - 1); };
                auto body = [&](int i, auto parity, bool more) {
                    constexpr int j = decltype(parity)::value;
                    floatx4 l;
                    if (AHEAD == 2) read_tile(place(i + 1), Qs[1 - j], l);
                    scores(Qs[AHEAD == 2 ? j : 0], Ss[j]);
                    if (AHEAD == 1) read_tile(place(i + 1), Qs[0], l);
                    if (more) add_weights(0, Ss[1 - j], ls[1 - j], 0, false);
                    ls[1 - j] = l;
                };
                // (of a SIMD's two waves the older one is served first, and the other is what the block's barrier waits for: 508 us, so 501)
                if (wave >= WAVES / 2) __builtin_amdgcn_s_setprio(1);
                read_tile(place(0), Qs[0], ls[0]);
                // (the last tile's logarithm is still wanted: ls[1] moves on only in the first body)
                if (pending) {
                    body(0, std::integral_constant<int, 0>(), true);
                    interleave<0, ND>();
                } else {
                    body(0, std::integral_constant<int, 0>(), false);
                }
                body(1, std::integral_constant<int, 1>(), true);
                interleave<0, ND>();
#pragma unroll 1
                for (int i = 2; i < TILES; i += 2) {
                    if (2 * i >= TILES) __builtin_amdgcn_s_setprio(0);
                    body(i, std::integral_constant<int, 0>(), true);
                    interleave<0, ND>();
                    body(i + 1, std::integral_constant<int, 1>(), true);
                    interleave<0, ND>();
                }
                pending = true;
                return;
            }
            if (STREAM) flush();
            if (masked) {
#pragma unroll 1
                for (int i = row_wave; i < count; i += row_waves) add_tile(tile + i, u0, true);
            } else {
#pragma unroll 1
                for (int i = row_wave; i < count; i += row_waves) add_tile(tile + i, u0, false);
            }
        };
        if constexpr (STREAM) {
            // queries that see any of the workgroup's tokens of this step
            const int i_lo = a.causal ? min(max(step - base, 0), nq) : 0;
            const int i_hi = a.window ? (int)max(min((int64_t)nq, (int64_t)min(step + step_tokens, end) - 1 + a.window - base), (int64_t)i_lo) : nq;
            int r_lo = i_lo * A.group.by, r_hi = i_hi * A.group.by;
            if (divided) {                                        // this workgroup's blocks of rows
                const int each = ((r_hi - r_lo + A.block_rows - 1) / A.block_rows + A.splits - 1) / A.splits * A.block_rows;
                r_lo = (int)min((int64_t)r_lo + (int64_t)split * each, (int64_t)r_hi);
                r_hi = (int)min((int64_t)r_lo + each, (int64_t)r_hi);
            }
            if (!idle) {
                place_rows(r_lo);
                ask_rows(r_lo, r_hi);
            }
            __syncthreads();                                      // (the table is there, the last step's rows are done with)
            if (!idle) decode(0);
            if (more) ask(t0 + step_tokens);
            if (!idle) put_rows(0);
            for (int r0 = r_lo, buffer = 0; r0 < r_hi; r0 += A.block_rows, buffer ^= 1) {
                const int r1 = min(r0 + A.block_rows, r_hi);
                __syncthreads();
                hushed = muted(buffer);
                if (r1 < r_hi) {
                    if (!A.whole_tokens) place_rows(r1);
                    ask_rows(r1, r_hi);
                }
                if (some) add_tiles(buffer * TILES, (r1 - r0 + 15) / 16, r0, r1, 0);
                if (r1 < r_hi) put_rows(buffer ^ 1);
            }
            flush();
        } else if (some) {
#pragma unroll
            for (int u0 = 0; u0 < 4; u0 += HOLD) {
                decode(u0);
                if (u0 + HOLD == 4 && more) ask(t0 + step_tokens);
                if (tiles) add_tiles(0, tiles, 0, rows, u0);
            }
        }
        float sum = add_rows(acc[0], acc[1], acc[2], acc[3]);     // of token t0 + lane
        if (row_waves > 1) {
            __syncthreads();
            parts[wave][lane] = sum;
            __syncthreads();
            if (row_wave == 0)
                for (int w = 1; w < row_waves; ++w) sum += parts[w * token_waves + token_wave][lane];
        }
        if (row_wave || lane >= TOKENS || t0 + lane >= end) continue;
        if (divided) A.a.part[((int64_t)unit * A.splits + split) * A.bound + t0 + lane] = sum;
        else if (to >= 0) a.out[to] = t0 + lane < known ? fmaf(a.decay, was, sum) : sum;
    }
}

// Adds the parts of divided rows, in their order.
__global__ __launch_bounds__(256) void kv_weigh_join_kernel(WeighArgs A) {
    const KVWeigh& a = A.a;
    const KVView& c = A.c;
    const int units = c.heads * a.B, unit = blockIdx.x % units, h = unit % c.heads, b = unit / c.heads;
    const int64_t t = (int64_t)(blockIdx.x / units) * 256 + threadIdx.x;
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    if (t >= min((int64_t)len, A.bound)) return;
    const int page = a.pages[(int64_t)b * a.max_pages + (t >> c.page_shift)];
    if (page < 0 || page >= c.pages) return;
    const int64_t at = (((int64_t)page * c.heads + h) << c.page_shift) + (t & ((1 << c.page_shift) - 1));
    const float* part = a.part + (int64_t)unit * A.splits * A.bound + t;
    float sum = 0.f;
#pragma unroll 4
    for (int s = 0; s < A.splits; ++s) sum += part[s * A.bound];
    a.out[at] = t < (a.known ? a.known[b] : len) ? fmaf(a.decay, a.mass[at], sum) : sum;
}

KVWeighPlan choose_weigh_plan(const KVView& c, int q_heads, int B, int max_q, int64_t max_len) {
    const int ND = c.d / 32;
    const int64_t rows = (int64_t)max_q * (q_heads / c.heads), units = device_cu_count(), tiles = cdiv(rows, 16);
    KVWeighPlan p;
    p.stream = rows > 2 * block_rows(ND, false);
    p.row_waves = p.splits = 1;
    const int tokens = weigh_tokens(ND, p.stream), most = std::min(kWeighWaves / 2, block_rows(ND, p.stream) / 16);
    // Waves share their tokens and divide the rows where tokens alone do not fill the chip.  8 heads of 128, 32 queries of 4 heads, one sequence of 1000
    // tokens: each its own 10.3 us, two share 7.8, four 6.5; of 20000: 13.4 and 18.4.
    while (!p.stream && 2 * p.row_waves <= most && tiles >= 4 * p.row_waves && cdiv(max_len, tokens * kWeighWaves / p.row_waves) * B * c.heads < units)
        p.row_waves *= 2;
    const int64_t step = tokens * kWeighWaves / p.row_waves, steps = cdiv(max_len, step), all = steps * B * c.heads;
    // Steps of a workgroup: up to four, as long as there are four workgroups to a compute unit.  64 sequences of up to 8192: one 62 us, two 54, four 51, eight 54;
    // 6 x 32 queries over up to 15000: one 18, two 22, four 29.
    p.chunk = (p.stream ? 1 : std::min((int64_t)4, std::max((int64_t)1, all / (4 * units)))) * step;
    p.blocks = (int)cdiv(max_len, p.chunk);
    if (p.stream) {
        // Four workgroups to a compute unit, one after the other: the first tokens are seen by all queries, the last by few, and workgroups of all
        // rows end unevenly.  2 x 4096 queries over up to 9000 tokens: all rows 537 us, four to a unit 514, eight 528; 8 x 1024 rows
        // of 256 channels over 1024 tokens 550 and 25.
        p.splits = (int)std::max((int64_t)1, std::min({cdiv(4 * units, all), cdiv(rows, block_rows(ND, true)), (int64_t)64}));
    }
    return p;
}

template <bool BF, int ND>
static void launch_width(const WeighArgs& A, const KVWeighPlan& p, hipStream_t s) {
    const unsigned grid = (unsigned)((int64_t)p.blocks * p.splits * A.c.heads * A.a.B);
    if (p.stream) kv_weigh_kernel<BF, ND, true><<<grid, kWeighThreads, 0, s>>>(A);
    else kv_weigh_kernel<BF, ND, false><<<grid, kWeighThreads, 0, s>>>(A);
}

template <bool BF>
static fk_status launch_weigh(const WeighArgs& A, const KVWeighPlan& p, hipStream_t s) {
    switch (A.c.d / 32) {
        case 1: launch_width<BF, 1>(A, p, s); break;
        case 2: launch_width<BF, 2>(A, p, s); break;
        case 3: launch_width<BF, 3>(A, p, s); break;
        case 4: launch_width<BF, 4>(A, p, s); break;
        case 5: launch_width<BF, 5>(A, p, s); break;
        case 6: launch_width<BF, 6>(A, p, s); break;
        case 7: launch_width<BF, 7>(A, p, s); break;
        default: launch_width<BF, 8>(A, p, s); break;
    }
    FK_HIP(hipGetLastError());
    return FK_OK;
}

fk_status launch_kv_weigh(const KVView& c, const KVWeigh& a, const KVWeighPlan& p, hipStream_t s) {
    const int64_t units = (int64_t)c.heads * a.B, bound = p.blocks * p.chunk;
    if (p.blocks * p.splits * units > UINT32_MAX / kWeighThreads) {
        set_error("fk_kv_weigh: unsupported size: %lld workgroups", (long long)(p.blocks * p.splits * units));
        return FK_EUNSUPPORTED;
    }
    const int group = a.q_heads / c.heads, room = block_rows(c.d / 32, p.stream);
    const bool whole = p.stream && group <= room;
    const WeighArgs A{c, a, Divider(group), p.row_waves, p.blocks, p.splits, bound, whole ? room / group * group : room, whole ? room / group : 0, whole, p.chunk, a.scale * 1.44269504088896341f};
    FK_TRY(c.bf ? launch_weigh<true>(A, p, s) : launch_weigh<false>(A, p, s));
    if (p.splits > 1) {
        kv_weigh_join_kernel<<<(unsigned)(units * cdiv(bound, 256)), 256, 0, s>>>(A);
        FK_HIP(hipGetLastError());
    }
    return FK_OK;
}

}  // namespace fk
