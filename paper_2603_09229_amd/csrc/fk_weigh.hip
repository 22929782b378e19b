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

constexpr int kWeighWaves = 8;
constexpr int kWeighTokens = 64;         // tokens a wave holds

struct WeighArgs {
    KVView c;
    KVWeigh a;
    Divider group;
    int row_waves;
    int64_t chunk;
    float scale_log2;
};

// sum over the 16 lanes of a row
__device__ __forceinline__ float add_columns(float x) {
    auto turn = [](float v, auto by) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), by(), 0xf, 0xf, false)); };
    x += turn(x, [] { return 0x128; });
    x += turn(x, [] { return 0x124; });
    x += turn(x, [] { return 0x122; });
    x += turn(x, [] { return 0x121; });
    return x;
}

template <bool BF, int ND>
__global__ __launch_bounds__(64 * kWeighWaves, 2) void kv_weigh_kernel(WeighArgs A) {
    using T = Table;
    __shared__ __align__(16) uint8_t lds[T::bytes];
    const KVWeigh& a = A.a;
    const KVView& c = A.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
    const int h = blockIdx.y, b = blockIdx.z;
    const int token_waves = kWeighWaves / A.row_waves, token_wave = wave & (token_waves - 1), row_wave = wave / token_waves;
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    const int64_t begin = blockIdx.x * A.chunk, end = blockIdx.x + 1 == gridDim.x ? len : min((int64_t)len, begin + A.chunk);
    if (begin >= len) return;
    const int q0 = a.q_start ? min(max(a.q_start[b], 0), (int)a.Tq) : b * a.max_q;
    const int nq = a.q_start ? min(min(max(a.q_start[b + 1] - q0, 0), a.max_q), (int)a.Tq - q0) : a.max_q;
    const int known = a.known ? a.known[b] : len, base = len - nq;
    T::fill<BF, 64 * kWeighWaves>(lds, T::level(c, h, lane), lane);
    __syncthreads();
    const uint32_t copy = (lane & 31) * 4;
    const int32_t* table = a.pages + (int64_t)b * a.max_pages;
    const int last_part = (a.max_pages << c.page_shift) - 16;
    auto row_of = [&](int at) {                                   // the cache's row of token `at`, in one of the table's pages
        const int page = min(max(table[min(at, last_part) >> c.page_shift], 0), (int)c.pages - 1);
        return (((int64_t)page * c.heads + h) << c.page_shift) + (min(at, last_part + 15) & ((1 << c.page_shift) - 1));
    };

    for (int64_t step = begin; step < end; step += kWeighTokens * token_waves) {
        const int t0 = (int)step + token_wave * kWeighTokens;
        float acc[4][4] = {};
        if (t0 < end) {
            uintx4 K[4][ND];
            float ks[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t row = row_of(t0 + 16 * u) & ~(int64_t)15;
                const uint32_t* codes = (const uint32_t*)(c.k_codes + (row + n) * (16 * ND) + q * (4 * ND));
#pragma unroll
                for (int k = 0; k < ND; ++k) {
                    const uint32_t w = codes[k];
#pragma unroll
                    for (int j = 0; j < 4; ++j) K[u][k][j] = T::pair<false>(lds, w, j, copy);
                }
                const uintx2 s = *(const uintx2*)(c.k_scale + row + 4 * q);
#pragma unroll
                for (int r = 0; r < 4; ++r) ks[u][r] = scale_at<BF>(s, r) * A.scale_log2;
            }
            // queries that see any of these tokens
            const int i_lo = a.causal ? min(max(t0 - base, 0), nq) : 0;
            const int i_hi = a.window ? max(min((int64_t)nq, (int64_t)t0 + kWeighTokens - 1 + a.window - base), (int64_t)i_lo) : nq;
            const int r_hi = i_hi * A.group.by;
            for (int r0 = i_lo * A.group.by + 16 * row_wave; r0 < r_hi; r0 += 16 * A.row_waves) {
                const int row = r0 + n, i = A.group.quotient(row), g = row - i * A.group.by;
                const bool live = row < r_hi;
                const int64_t token = q0 + (live ? i : 0);
                const int head = h * A.group.by + (live ? g : 0);
                const uint16_t* at = a.q.at + token * a.q.token + (int64_t)head * a.q.head + q * (8 * ND);
                uintx4 Q[ND];
#pragma unroll
                for (int k = 0; k < ND; ++k) Q[k] = *(const uintx4_any*)(at + 8 * k);
                float lse = a.lse[token * a.q_heads + head] * 1.44269504088896341f;
                lse = live && lse != -INFINITY ? lse : INFINITY;
                const int pos = base + i, p0 = base + A.group.quotient(r0), p1 = base + A.group.quotient(min(r0 + 15, r_hi - 1));
                const bool masked = (a.causal && p0 < t0 + kWeighTokens - 1) || (a.window && t0 <= p1 - a.window);
                floatx4 S[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    S[u] = floatx4{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < ND; ++k) S[u] = mfma16<BF>(K[u][k], Q[k], S[u]);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float w = exp2_fast(fmaf(S[u][r], ks[u][r], -lse));
                        if (masked) {
                            const int t = t0 + 16 * u + 4 * q + r;
                            w = (a.causal && t > pos) || (a.window && t <= pos - a.window) ? 0.f : w;
                        }
                        acc[u][r] += w;
                    }
            }
        }
        float sum = 0.f;                                          // lane (n, q): token 16 (n / 4) + 4 q + n % 4
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = add_columns(acc[u][r]);
                sum = n == 4 * u + r ? x : sum;
            }
        if (A.row_waves > 1) {
            __shared__ float parts[kWeighWaves][kWeighTokens];
            __syncthreads();
            parts[wave][lane] = sum;
            __syncthreads();
            if (row_wave == 0)
                for (int w = 1; w < A.row_waves; ++w) sum += parts[w * token_waves + token_wave][lane];
        }
        const int t = t0 + 16 * (n >> 2) + 4 * q + (n & 3);
        if (row_wave == 0 && t < end) {
            const int64_t row = row_of(t);
            a.out[row] = t < known ? fmaf(a.decay, a.mass[row], sum) : sum;
        }
    }
}

KVWeighPlan choose_weigh_plan(const KVView& c, int q_heads, int B, int max_q, int64_t max_len) {
    const int64_t rows = (int64_t)max_q * (q_heads / c.heads), units = device_cu_count(), tiles = cdiv(rows, 16);
    KVWeighPlan p;
    p.row_waves = 1;
    while (p.row_waves < kWeighWaves && tiles >= 4 * p.row_waves && cdiv(max_len, kWeighTokens * kWeighWaves / p.row_waves) * B * c.heads < 2 * units)
        p.row_waves *= 2;
    const int64_t step = kWeighTokens * kWeighWaves / p.row_waves, steps = cdiv(max_len, step);
    const int64_t each = std::max((int64_t)1, steps * B * c.heads / (4 * units));
    p.chunk = (rows <= 64 ? each : 1) * step;
    p.blocks = (int)cdiv(max_len, p.chunk);
    return p;
}

template <bool BF>
static fk_status launch_weigh(const WeighArgs& A, const KVWeighPlan& p, hipStream_t s) {
    const dim3 grid(p.blocks, A.c.heads, A.a.B);
    const int threads = 64 * kWeighWaves;
    switch (A.c.d / 32) {
        case 1: kv_weigh_kernel<BF, 1><<<grid, threads, 0, s>>>(A); break;
        case 2: kv_weigh_kernel<BF, 2><<<grid, threads, 0, s>>>(A); break;
        case 3: kv_weigh_kernel<BF, 3><<<grid, threads, 0, s>>>(A); break;
        case 4: kv_weigh_kernel<BF, 4><<<grid, threads, 0, s>>>(A); break;
        case 5: kv_weigh_kernel<BF, 5><<<grid, threads, 0, s>>>(A); break;
        case 6: kv_weigh_kernel<BF, 6><<<grid, threads, 0, s>>>(A); break;
        case 7: kv_weigh_kernel<BF, 7><<<grid, threads, 0, s>>>(A); break;
        default: kv_weigh_kernel<BF, 8><<<grid, threads, 0, s>>>(A); break;
    }
    FK_HIP(hipGetLastError());
    return FK_OK;
}

fk_status launch_kv_weigh(const KVView& c, const KVWeigh& a, const KVWeighPlan& p, hipStream_t s) {
    const WeighArgs A{c, a, Divider(a.q_heads / c.heads), p.row_waves, p.chunk, a.scale * 1.44269504088896341f};
    return c.bf ? launch_weigh<true>(A, p, s) : launch_weigh<false>(A, p, s);
}

}  // namespace fk
