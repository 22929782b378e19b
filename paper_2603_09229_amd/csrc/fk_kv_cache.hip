// Rows into and out of the 4-bit key/value cache.
//
// Coding a row x of d numbers: s = max |x|, id = the level l nearest to x / s.  With levels in ascending order
// that is the number of middles m_j = (l_j + l_{j+1}) / 2 below x / s, found in four steps of a binary search;
// x / s > m_j is asked as x - s m_j > 0, one fused multiply-add whose sign is the exact one.  The largest
// magnitude is found on the 16 bits themselves: without the sign they order as integers, values that are not finite last.
//
// A row is held by L lanes of a wave, 8 channels (16 bytes) each, so that rows of 64 / L heads move together.
//
// What bounds it: bytes for many tokens (16384 of 8 + 8 + 32 rows of 128: 361 MB in 74 us one call after the other, 80 by the profiler, 4.9 and 4.5 TB/s,
// where a large copy reaches 5.2; reading 20000 tokens of 8 + 8 rows of 128: 103 MB in 23 us, 4.5), the launch and three dependent loads for
// few (3.8 and 2.1 us for one token), the latency of one round of workgroups between (4099 tokens of 4 + 4 + 24 rows of 64: 13 us).
#include "fk_device.h"
#include "fk_kv.h"

namespace fk {

constexpr int kAppendThreads = 256;
constexpr int kAhead = 2;                // groups of rows whose loads are on their way

// middles of the levels of all heads, keys then values: [2][heads][16] (the last is unused)
__device__ void middles_to_lds(const KVView& c, float* mid) {
    for (int i = threadIdx.x; i < 2 * c.heads * 16; i += blockDim.x) {
        const uint16_t* l = i < c.heads * 16 ? c.k_levels + i : c.v_levels + (i - c.heads * 16);
        mid[i] = (i & 15) < 15 ? 0.5f * (lp_to_float(l[0], c.bf) + lp_to_float(l[1], c.bf)) : 0.f;
    }
}

struct Angles {
    float cos[8], sin[8];          // of the lane's 8 channels; sin with the sign of the partner's term
};

__device__ __forceinline__ Angles load_angles(const KVAppend& a, int64_t token, int e0) {
    Angles t;
    const int p = min(max((int64_t)a.positions[token], (int64_t)0), a.max_pos - 1);
    const float* row = a.cos_sin + (int64_t)p * a.rot;
    const int half = a.rot / 2;
    if (e0 >= a.rot) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { t.cos[i] = 1.f; t.sin[i] = 0.f; }
        return t;
    }
    if (a.interleaved) {
        const floatx4 c = *(const floatx4*)(row + e0 / 2), s = *(const floatx4*)(row + half + e0 / 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.cos[i] = c[i / 2];
            t.sin[i] = i & 1 ? s[i / 2] : -s[i / 2];
        }
    } else {
        const bool first = e0 < half;
        const int q = first ? e0 : e0 - half;
        const floatx4 c0 = *(const floatx4*)(row + q), c1 = *(const floatx4*)(row + q + 4);
        const floatx4 s0 = *(const floatx4*)(row + half + q), s1 = *(const floatx4*)(row + half + q + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = i < 4 ? s0[i & 3] : s1[i & 3];
            t.cos[i] = i < 4 ? c0[i & 3] : c1[i & 3];
            t.sin[i] = first ? -s : s;
        }
    }
    return t;
}

// The lane's 8 channels turned.  Products and their sum are rounded one by one, as elementary operations round them.
template <bool BF>
__device__ __forceinline__ uintx4 turned(uintx4 x, const Angles& t, const KVAppend& a, int e0) {
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63, half = a.rot / 2;
    uintx4 y;                                                   // the partners' 8 channels
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (x[i] >> 16) | (x[i] << 16);
    } else {
        const int from = e0 >= a.rot ? lane : e0 < half ? lane + half / 8 : lane - half / 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __shfl((int)x[i], from);
    }
    uintx4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float z[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float u = lp_to_float((uint16_t)(x[i] >> 16 * h), BF) * t.cos[2 * i + h];
            const float v = lp_to_float((uint16_t)(y[i] >> 16 * h), BF) * t.sin[2 * i + h];
            z[h] = u + v;
        }
        r[i] = pack_lp<BF>(z[0], z[1]);
    }
    return e0 < a.rot ? r : x;
}

// 8 ids of the lane's channels, 4 bits each, and the row's scale (16 bits).  The first two steps' middles are in registers, the others are
// looked up.
template <bool BF, int L>
__device__ __forceinline__ uint32_t coded(uintx4 x, const float* mid, uint16_t* scale) {
    const float m3 = mid[3], m7 = mid[7], m11 = mid[11];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
#pragma unroll
    for (int o = 1; o < L; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const bool finite = top < (BF ? 0x7f80u : 0x7c00u);
    *scale = finite ? (uint16_t)top : (uint16_t)0x7fffu;
    const float s = -lp_to_float((uint16_t)top, BF);
    uint32_t ids = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = lp_to_float((uint16_t)(x[e / 2] >> 16 * (e & 1)), BF);
        const bool half = __fmaf_rn(s, m7, v) > 0.f;
        int id = half ? 8 : 0;
        id += __fmaf_rn(s, half ? m11 : m3, v) > 0.f ? 4 : 0;
        id += __fmaf_rn(s, mid[id + 1], v) > 0.f ? 2 : 0;
        id += __fmaf_rn(s, mid[id], v) > 0.f ? 1 : 0;
        ids |= (uint32_t)id << 4 * e;
    }
    return finite ? ids : 0;
}

// A unit of work: `per_unit` groups of rows of one token; a group is 64 / L heads of the keys, the values or the queries.  Units of
// whole tokens load the token's angles once.
template <bool BF, int L>
__global__ __launch_bounds__(kAppendThreads, 6) void kv_append_kernel(KVView c, KVAppend a, int per_unit) {
    extern __shared__ float mid[];
    constexpr int rows = 64 / L;
    const int lane = threadIdx.x & 63, e0 = (lane % L) * 8, sub = lane / L;
    const int kv_groups = (c.heads + rows - 1) / rows, q_groups = (a.q_heads + rows - 1) / rows;
    const int groups = 2 * kv_groups + q_groups, units = (groups + per_unit - 1) / per_unit;
    const int64_t waves = (int64_t)gridDim.x * (kAppendThreads / 64), all = a.T * units;
    const int64_t wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kAppendThreads / 64) + threadIdx.x / 64));
    bool first = true;
    for (int64_t u = wave;; u += waves, first = false) {
        const bool some = u < all;
        const int64_t token = some ? u / units : 0;
        const int g0 = some ? (int)(u - token * units) * per_unit : 0, g1 = some ? min(g0 + per_unit, groups) : g0;
        // rows of a group: keys, values or queries
        auto load = [&](int g) {
            const bool is_k = g < kv_groups, is_q = g >= 2 * kv_groups;
            const int head = (is_k ? g : is_q ? g - 2 * kv_groups : g - kv_groups) * rows + sub;
            const KVRows& from = is_k ? a.k : is_q ? a.q : a.v;
            uintx4 x = {0, 0, 0, 0};
            if (e0 < c.d && head < (is_q ? a.q_heads : c.heads))
                x = *(const uintx4_any*)(from.at + token * from.token + head * from.head + e0);
            return x;
        };
        uintx4 next[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i] = g0 + i < g1 ? load(g0 + i) : uintx4{0, 0, 0, 0};
        Angles t;
        if (a.rot) t = load_angles(a, token, e0);
        const int64_t slot = a.slots[token];
        if (first) {                                              // (the first unit's loads are on their way meanwhile)
            middles_to_lds(c, mid);
            __syncthreads();
        }
        if (!some) break;
        const bool kept = slot >= 0 && (slot >> c.page_shift) < c.pages;
        const int64_t place = (((slot >> c.page_shift) * c.heads) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
        for (int g = g0; g < g1; g += kAhead) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (g + i >= g1) break;
                uintx4 x = next[i];
                if (g + i + kAhead < g1) next[i] = load(g + i + kAhead);
                const bool is_k = g + i < kv_groups, is_q = g + i >= 2 * kv_groups;
                const int head = (is_k ? g + i : is_q ? g + i - 2 * kv_groups : g + i - kv_groups) * rows + sub;
                const bool live = e0 < c.d && head < (is_q ? a.q_heads : c.heads);
                if (a.rot && (is_k || is_q)) x = turned<BF>(x, t, a, e0);
                if (is_q) {
                    if (live) *(uintx4*)(a.q_out + (token * a.q_heads + head) * c.d + e0) = x;
                    continue;
                }
                uint16_t scale;
                const uint32_t ids = coded<BF, L>(x, mid + ((is_k ? 0 : c.heads) + min(head, c.heads - 1)) * 16, &scale);
                if (!live || !kept) continue;
                const int64_t row = place + ((int64_t)head << c.page_shift);
                *(uint32_t*)((is_k ? c.k_codes : c.v_codes) + row * (c.d / 2) + e0 / 2) = ids;
                if (e0 == 0) (is_k ? c.k_scale : c.v_scale)[row] = scale;
            }
        }
    }
}

template <bool BF, int L>
__global__ __launch_bounds__(kAppendThreads) void kv_read_kernel(KVView c, const int64_t* slots, int64_t T, uint16_t* k_out,
                                                                 uint16_t* v_out) {
    extern __shared__ float level[];                            // [2][heads][16]
    for (int i = threadIdx.x; i < 2 * c.heads * 16; i += blockDim.x)
        level[i] = lp_to_float(i < c.heads * 16 ? c.k_levels[i] : c.v_levels[i - c.heads * 16], c.bf);
    __syncthreads();
    constexpr int rows = 64 / L;
    const int lane = threadIdx.x & 63, e0 = (lane % L) * 8, sub = lane / L;
    const int groups = (c.heads + rows - 1) / rows;
    const int64_t waves = (int64_t)gridDim.x * (kAppendThreads / 64), all = T * groups * 2;
    const int64_t wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kAppendThreads / 64) + threadIdx.x / 64));
    for (int64_t u = wave; u < all; u += waves) {
        const int64_t token = u / (2 * groups);
        const int g = (int)(u - token * 2 * groups);
        const bool is_k = g < groups;
        uint16_t* out = is_k ? k_out : v_out;
        const int head = (is_k ? g : g - groups) * rows + sub;
        if (!out || e0 >= c.d || head >= c.heads) continue;
        const int64_t slot = slots[token];
        uintx4 r = {0, 0, 0, 0};
        if (slot >= 0 && (slot >> c.page_shift) < c.pages) {
            const int64_t row = (((slot >> c.page_shift) * c.heads + head) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
            const uint32_t ids = *(const uint32_t*)((is_k ? c.k_codes : c.v_codes) + row * (c.d / 2) + e0 / 2);
            const float s = lp_to_float((is_k ? c.k_scale : c.v_scale)[row], BF);
            const float* l = level + ((is_k ? 0 : c.heads) + head) * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = pack_lp<BF>(l[(ids >> 8 * i) & 15] * s, l[(ids >> (8 * i + 4)) & 15] * s);
        }
        *(uintx4*)(out + (token * c.heads + head) * c.d + e0) = r;
    }
}

static int lanes_of(int d) { return d <= 32 ? 4 : d <= 64 ? 8 : d <= 128 ? 16 : 32; }

// Waves for all units, but no more workgroups than the chip holds at once (`each` to a compute unit): the rest is done in turns, so that
// the levels are loaded once.  16384 tokens of 8 + 8 + 32 rows of 128: 6 to a unit 74 us, 8 (of which 6 run first, then 2) 81.
static unsigned grid_for(int64_t units, int each) {
    const int64_t blocks = cdiv(units, kAppendThreads / 64), most = (int64_t)device_cu_count() * each;
    return (unsigned)(blocks < most ? blocks : most);
}

fk_status launch_kv_append(const KVView& c, const KVAppend& a, hipStream_t s) {
    const int L = lanes_of(c.d), rows = 64 / L;
    const int64_t groups = 2 * cdiv(c.heads, rows) + cdiv(a.q_heads, rows);
    const int per_unit = a.T * groups <= (int64_t)device_cu_count() * 32 ? 1 : (int)groups;
    const unsigned grid = grid_for(a.T * cdiv(groups, per_unit), 6);
    const size_t lds = (size_t)c.heads * 16 * 2 * sizeof(float);
    auto kern = c.bf ? (L == 4 ? kv_append_kernel<true, 4> : L == 8 ? kv_append_kernel<true, 8>
                        : L == 16 ? kv_append_kernel<true, 16> : kv_append_kernel<true, 32>)
                     : (L == 4 ? kv_append_kernel<false, 4> : L == 8 ? kv_append_kernel<false, 8>
                        : L == 16 ? kv_append_kernel<false, 16> : kv_append_kernel<false, 32>);
    kern<<<grid, kAppendThreads, lds, s>>>(c, a, per_unit);
    FK_HIP(hipGetLastError());
    return FK_OK;
}

fk_status launch_kv_read(const KVView& c, const int64_t* slots, int64_t T, uint16_t* k_out, uint16_t* v_out, hipStream_t s) {
    const int L = lanes_of(c.d);
    const unsigned grid = grid_for(T * 2 * cdiv(c.heads, 64 / L), 8);
    const size_t lds = (size_t)c.heads * 16 * 2 * sizeof(float);
    auto kern = c.bf ? (L == 4 ? kv_read_kernel<true, 4> : L == 8 ? kv_read_kernel<true, 8>
                        : L == 16 ? kv_read_kernel<true, 16> : kv_read_kernel<true, 32>)
                     : (L == 4 ? kv_read_kernel<false, 4> : L == 8 ? kv_read_kernel<false, 8>
                        : L == 16 ? kv_read_kernel<false, 16> : kv_read_kernel<false, 32>);
    kern<<<grid, kAppendThreads, lds, s>>>(c, slots, T, k_out, v_out);
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
