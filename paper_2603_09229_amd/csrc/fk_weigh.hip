// Attention weights of cached tokens, added up over queries.
//
// w_t = (t known ? decay w_t : 0) + sum over query rows n that see t of 2^(scale log2 e s_t (q_n . K_t) - log2 e lse_n), a row being one head of
// the group at one query token, s_t the key's scale, lse_n the logarithm of the row's softmax sum, which attention has left.  No maximum is
// searched: the logarithm brings the weights to at most 1.
//
// A wave holds the keys of 64 tokens as operands of 16x16x32 MFMA, S^T = K q^T with tokens on the row side, and goes over the query rows 16 at
// a time.  A lane owns one column (query row) and 16 tokens of it, whose weights it adds up in registers; the 16 columns are added once at
// the end, in a fixed order.  Tokens belong to one workgroup, so nothing is added with atomics and the result does not depend on
// the order of workgroups.
#include <algorithm>

#include "fk_device.h"
#include "fk_evict.h"
#include "fk_kv_attend.h"

namespace fk {

constexpr int kWeighWaves = 8, kWeighThreads = 64 * kWeighWaves;
constexpr int kWeighTokens = 64;         // tokens a wave takes at a time

// Rows of queries in one of the two buffers, whole tiles; both together are all that a workgroup keeps.
constexpr int block_rows(int ND) { return 256 / ND / 16 * 16; }

struct WeighArgs {
    KVView c;
    KVWeigh a;
    Divider group;
    int row_waves;
    int64_t chunk;
    float scale_log2;
};

// LDS: the table of pairs of the keys' levels, 256 rows of 32 copies, in the lower halves of rows of 256 bytes (a byte of codes is then the
// address with one v_perm), and the queries in the upper ones, in the order in which a wave's lanes read them as operands, 16 bytes a lane.
// Lanes that write a row's pieces meet in a bank unless the rows' order within a piece's slot is turned by the piece.
struct WeighLds {
    static constexpr int bytes = 65536;
    static __device__ __forceinline__ int slot_byte(int slot) { return (slot >> 3) * 256 + 128 + (slot & 7) * 16; }
    // piece k of quarter q of row n of a tile
    template <int ND>
    static __device__ __forceinline__ int piece(int tile, int k, int q, int n) {
        return slot_byte((tile * ND + k) * 64 + q * 16 + (n ^ (((q * 4) ^ k) & 15)));
    }
    static __device__ __forceinline__ void fill(uint8_t* lds, uint16_t level) {
#pragma unroll
        for (int i = 0; i < 256 * 8 / kWeighThreads; ++i) {
            const int at = i * kWeighThreads + threadIdx.x, code = at / 8;
            const uint32_t pair = (uint32_t)__shfl((int)level, code & 15) | ((uint32_t)__shfl((int)level, code >> 4) << 16);
            *(uintx4*)(lds + code * 256 + (at & 7) * 16) = uintx4{pair, pair, pair, pair};
        }
    }
};

// the upper halves of the first and the lower halves of the second register change places, in units of BY lanes
template <int BY>
__device__ __forceinline__ void swap_lanes(float& a, float& b) {
    typedef uint32_t uintx2v __attribute__((ext_vector_type(2)));
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

// STREAM: more query rows than a workgroup keeps; they come by in two buffers, once for every step of tokens.
template <bool BF, int ND, bool STREAM>
__global__ __launch_bounds__(kWeighThreads, !STREAM && ND <= 4 ? 4 : 2) void kv_weigh_kernel(WeighArgs A) {
    constexpr int HB = block_rows(ND), PIECES = HB * 4 * ND, EACH = (PIECES + kWeighThreads - 1) / kWeighThreads;
    constexpr int HOLD = STREAM ? 4 : 2;                          // 16 tokens each, whose keys are operands at the same time
    __shared__ __align__(16) uint8_t lds[WeighLds::bytes];
    __shared__ __align__(16) float logs[2 * HB];                  // of a row: its logarithm in powers of two,
    __shared__ __align__(16) int upto[2 * HB], from[2 * HB];      // and it sees the tokens behind `from` up to `upto`
    __shared__ float parts[kWeighWaves][kWeighTokens];
    const KVWeigh& a = A.a;
    const KVView& c = A.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int h = blockIdx.y, b = blockIdx.z;
    const uint16_t level = c.k_levels[h * 16 + n];
    const int token_waves = kWeighWaves / A.row_waves, token_wave = wave & (token_waves - 1), row_wave = wave / token_waves;
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    const int64_t begin64 = blockIdx.x * A.chunk;
    if (begin64 >= len) return;                                   // the whole workgroup
    const int begin = (int)begin64, end = blockIdx.x + 1 == gridDim.x ? len : (int)min((int64_t)len, begin64 + A.chunk);
    const int q0 = a.q_start ? min(max(a.q_start[b], 0), (int)a.Tq) : b * a.max_q;
    const int nq = a.q_start ? min(min(max(a.q_start[b + 1] - q0, 0), a.max_q), (int)a.Tq - q0) : a.max_q;
    const int known = a.known ? a.known[b] : len, base = len - nq, rows = nq * A.group.by;
    const int step_tokens = kWeighTokens * token_waves;

    // A wave's tokens: page of token t0 + lane, codes, scales and weights so far, one step ahead.
    const int32_t* table = a.pages + (int64_t)b * a.max_pages;
    const int last = (a.max_pages << c.page_shift) - 1;
    int page;
    uint32_t codes[4][ND];
    uint16_t scale;
    float old;
    int64_t at;                                                   // the cache's row of token t0 + lane
    auto ask_page = [&](int t0) { page = table[min(t0 + lane, last) >> c.page_shift]; };
    auto ask = [&](int t0) {
        page = min(max(page, 0), (int)c.pages - 1);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int p = __builtin_amdgcn_readlane(page, 16 * u), first = min(t0 + 16 * u, last - 15) & ((1 << c.page_shift) - 1);
            const Base base = base_of(c.k_codes, ((((int64_t)p * c.heads + h) << c.page_shift) + first) * (16 * ND));
#pragma unroll
            for (int k = 0; k < ND; ++k) codes[u][k] = load_at<uint32_t>(base, n * (16 * ND) + q * (4 * ND) + 4 * k);
        }
        at = (((int64_t)page * c.heads + h) << c.page_shift) + (min(t0 + lane, last) & ((1 << c.page_shift) - 1));
        scale = c.k_scale[at];
        old = t0 + lane < min(known, end) ? a.mass[at] : 0.f;
    };
    ask_page(begin + token_wave * kWeighTokens);

    // Rows of queries on their way into a buffer.
    uintx4 piece[EACH];
    float log_in = 0.f;
    int upto_in = 0, from_in = 0;
    auto ask_rows = [&](int row0, int r_hi) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int x = e * kWeighThreads + threadIdx.x, row = row0 + x / (4 * ND);
            piece[e] = uintx4{0, 0, 0, 0};
            if (x < PIECES && row < r_hi) {
                const int i = A.group.quotient(row), g = row - i * A.group.by;
                piece[e] = *(const uintx4_any*)(a.q.at + (int64_t)(q0 + i) * a.q.token + (int64_t)(h * A.group.by + g) * a.q.head + x % (4 * ND) * 8);
            }
        }
        if (threadIdx.x < HB) {
            const int row = row0 + threadIdx.x, i = A.group.quotient(row), g = row - i * A.group.by;
            log_in = INFINITY;                                    // (of a row that is none, or that has seen nothing: weights of 0)
            upto_in = -1;
            from_in = INT32_MAX;
            if (row < r_hi) {
                const float l = a.lse[(int64_t)(q0 + i) * a.q_heads + h * A.group.by + g] * 1.44269504088896341f;
                log_in = l == -INFINITY ? INFINITY : l;
                upto_in = a.causal ? base + i : INT32_MAX;
                from_in = a.window ? base + i - a.window : -1;
            }
        }
    };
    auto put_rows = [&](int buffer) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int x = e * kWeighThreads + threadIdx.x, row = x / (4 * ND), p = x % (4 * ND);
            if (x < PIECES) *(uintx4*)(lds + WeighLds::piece<ND>(buffer * (HB / 16) + row / 16, p % ND, p / ND, row & 15)) = piece[e];
        }
        if (threadIdx.x < HB) {
            logs[buffer * HB + threadIdx.x] = log_in;
            upto[buffer * HB + threadIdx.x] = upto_in;
            from[buffer * HB + threadIdx.x] = from_in;
        }
    };
    int tiles = 0;
    if constexpr (!STREAM) {
        tiles = (rows + 15) / 16;
        ask_rows(0, rows);
        put_rows(0);
        if (rows > HB) {
            ask_rows(HB, rows);
            put_rows(1);
        }
    }
    WeighLds::fill(lds, level);
    ask(begin + token_wave * kWeighTokens);
    if (!STREAM) __syncthreads();
    const uint32_t copy = (lane & 31) * 4;
    const int q_lane = WeighLds::piece<ND>(0, 0, q, n);           // (piece k: its bits 4 to 6 turned by k)

    for (int step = begin; step < end; step += step_tokens) {
        const int t0 = step + token_wave * kWeighTokens;
        const bool some = t0 < end;
        const int64_t to = at;
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
        // rows r0 .. r0 + 15, in place `tile` of the buffers
        auto add_tile = [&](int tile, int r0, int r_hi, int u0) {
            const int p0 = base + A.group.quotient(r0), p1 = base + A.group.quotient(min(r0 + 15, r_hi - 1));
            const int first = t0 + 16 * u0, final = first + 16 * HOLD - 1;
            if ((a.causal && p1 < first) || (a.window && final <= p0 - a.window)) return;   // no row sees any of these tokens
            const bool masked = (a.causal && p0 < final) || (a.window && first <= p1 - a.window);
            uintx4 Q[ND];
#pragma unroll
            for (int k = 0; k < ND; ++k) Q[k] = *(const uintx4*)(lds + (q_lane ^ (k * 16)) + (tile * ND + k) * 2048);
            const floatx4 l = *(const floatx4*)(logs + tile * 16 + 4 * q);
            floatx4 S[HOLD];
#pragma unroll
            for (int u = 0; u < HOLD; ++u) {
                S[u] = floatx4{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < ND; ++k) S[u] = mfma16<BF>(Q[k], K[u][k], S[u]);
            }
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
                        const int t = first + 16 * u + n;
                        w[u][r] = t <= hi[r] && t > lo[r] ? w[u][r] : 0.f;
                    }
            }
#pragma unroll
            for (int u = 0; u < HOLD; ++u) acc[u0 + u] += (w[u][0] + w[u][1]) + (w[u][2] + w[u][3]);
        };
        if constexpr (STREAM) {
            // queries that see any of the workgroup's tokens of this step
            const int i_lo = a.causal ? min(max(step - base, 0), nq) : 0;
            const int i_hi = a.window ? (int)max(min((int64_t)nq, (int64_t)min(step + step_tokens, end) - 1 + a.window - base), (int64_t)i_lo) : nq;
            const int r_lo = i_lo * A.group.by, r_hi = i_hi * A.group.by;
            ask_rows(r_lo, r_hi);
            __syncthreads();                                      // (the table is there, the last step's rows are done with)
            decode(0);
            if (more) ask(t0 + step_tokens);
            put_rows(0);
            for (int r0 = r_lo, buffer = 0; r0 < r_hi; r0 += HB, buffer ^= 1) {
                __syncthreads();
                if (r0 + HB < r_hi) ask_rows(r0 + HB, r_hi);
                if (some)
                    for (int tile = row_wave; tile < HB / 16 && r0 + 16 * tile < r_hi; tile += A.row_waves)
                        add_tile(buffer * (HB / 16) + tile, r0 + 16 * tile, r_hi, 0);
                if (r0 + HB < r_hi) put_rows(buffer ^ 1);
            }
        } else if (some) {
#pragma unroll
            for (int u0 = 0; u0 < 4; u0 += HOLD) {
                decode(u0);
                if (u0 + HOLD == 4 && more) ask(t0 + step_tokens);
                for (int tile = row_wave; tile < tiles; tile += A.row_waves) add_tile(tile, 16 * tile, rows, u0);
            }
        }
        float sum = add_rows(acc[0], acc[1], acc[2], acc[3]);     // of token t0 + lane
        if (A.row_waves > 1) {
            __syncthreads();
            parts[wave][lane] = sum;
            __syncthreads();
            if (row_wave == 0)
                for (int w = 1; w < A.row_waves; ++w) sum += parts[w * token_waves + token_wave][lane];
        }
        if (row_wave == 0 && t0 + lane < end) a.out[to] = t0 + lane < known ? fmaf(A.a.decay, was, sum) : sum;
    }
}

KVWeighPlan choose_weigh_plan(const KVView& c, int q_heads, int B, int max_q, int64_t max_len) {
    const int64_t rows = (int64_t)max_q * (q_heads / c.heads), units = device_cu_count(), tiles = cdiv(rows, 16);
    KVWeighPlan p;
    p.stream = rows > 2 * block_rows(c.d / 32);
    p.row_waves = 1;
    const int most = std::min(4, block_rows(c.d / 32) / 16);
    while (2 * p.row_waves <= most && tiles >= 4 * p.row_waves && cdiv(max_len, kWeighTokens * kWeighWaves / p.row_waves) * B * c.heads < 2 * units)
        p.row_waves *= 2;
    const int64_t step = kWeighTokens * kWeighWaves / p.row_waves, steps = cdiv(max_len, step);
    const int64_t each = std::min((int64_t)4, std::max((int64_t)1, steps * B * c.heads / (4 * units)));
    p.chunk = (p.stream ? 1 : each) * step;
    p.blocks = (int)cdiv(max_len, p.chunk);
    return p;
}

template <bool BF, int ND>
static void launch_width(const WeighArgs& A, const KVWeighPlan& p, hipStream_t s) {
    const dim3 grid(p.blocks, A.c.heads, A.a.B);
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
    const WeighArgs A{c, a, Divider(a.q_heads / c.heads), p.row_waves, p.chunk, a.scale * 1.44269504088896341f};
    return c.bf ? launch_weigh<true>(A, p, s) : launch_weigh<false>(A, p, s);
}

}  // namespace fk
