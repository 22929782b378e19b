// Rows into and out of the 4-bit key/value cache.
//
// Coding a row x of d numbers: s = max |x|, id = the level l nearest to x / s.  With levels in ascending order
// that is the number of middles m_j = (l_j + l_{j+1}) / 2 below x / s, found in four steps of a binary search;
// x / s > m_j is asked as x - s m_j > 0, one fused multiply-add whose sign is the exact one.  The largest
// magnitude is found on the 16 bits themselves: without the sign they order as integers, values that are not finite last.
//
// A row is held by L lanes of a wave, 8 channels (16 bytes) each, so that rows of 64 / L heads move together.
#include "fk_device.h"
#include "fk_kv.h"

namespace fk {

constexpr int kAppendThreads = 256;

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

template <int L>
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
template <int L>
__device__ __forceinline__ uintx4 turned(uintx4 x, const Angles& t, const KVAppend& a, int e0, bool bf) {
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
        uint32_t w = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float u = lp_to_float((uint16_t)(x[i] >> 16 * h), bf) * t.cos[2 * i + h];
            const float v = lp_to_float((uint16_t)(y[i] >> 16 * h), bf) * t.sin[2 * i + h];
            w |= (uint32_t)float_to_lp_any(u + v, bf) << 16 * h;
        }
        r[i] = w;
    }
    return e0 < a.rot ? r : x;
}

// 8 ids of the lane's channels, 4 bits each, and the row's scale (16 bits)
template <int L>
__device__ __forceinline__ uint32_t coded(uintx4 x, const float* mid, bool bf, uint16_t* scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
#pragma unroll
    for (int o = 1; o < L; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const bool finite = top < (bf ? 0x7f80u : 0x7c00u);
    *scale = finite ? (uint16_t)top : (uint16_t)0x7fffu;
    if (!finite) return 0;
    const float s = -lp_to_float((uint16_t)top, bf);
    uint32_t ids = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = lp_to_float((uint16_t)(x[e / 2] >> 16 * (e & 1)), bf);
        int id = 0;
#pragma unroll
        for (int step = 8; step; step /= 2) id += __fmaf_rn(s, mid[id + step - 1], v) > 0.f ? step : 0;
        ids |= (uint32_t)id << 4 * e;
    }
    return ids;
}

// A unit of work: `per_unit` groups of rows of one token; a group is 64 / L heads of the keys, the values or the queries.  Units of
// whole tokens load the token's angles once.
template <int L>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(KVView c, KVAppend a, int per_unit) {
    extern __shared__ float mid[];
    middles_to_lds(c, mid);
    __syncthreads();
    constexpr int rows = 64 / L;
    const int lane = threadIdx.x & 63, e0 = (lane % L) * 8, sub = lane / L;
    const int kv_groups = (c.heads + rows - 1) / rows, q_groups = (a.q_heads + rows - 1) / rows;
    const int groups = 2 * kv_groups + q_groups, units = (groups + per_unit - 1) / per_unit;
    const int64_t waves = (int64_t)gridDim.x * (kAppendThreads / 64), all = a.T * units;
    const int64_t wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kAppendThreads / 64) + threadIdx.x / 64));
    for (int64_t u = wave; u < all; u += waves) {
        const int64_t token = u / units;
        const int g0 = (int)(u - token * units) * per_unit, g1 = min(g0 + per_unit, groups);
        Angles t;
        if (a.rot) t = load_angles<L>(a, token, e0);
        const int64_t slot = a.slots[token];
        const bool kept = slot >= 0 && (slot >> c.page_shift) < c.pages;
        for (int g = g0; g < g1; ++g) {
            const bool is_k = g < kv_groups, is_q = g >= 2 * kv_groups;
            const int head = (is_k ? g : is_q ? g - 2 * kv_groups : g - kv_groups) * rows + sub;
            const KVRows& from = is_k ? a.k : is_q ? a.q : a.v;
            const bool live = e0 < c.d && head < (is_q ? a.q_heads : c.heads);
            uintx4 x = {0, 0, 0, 0};
            if (live) x = *(const uintx4_any*)(from.at + token * from.token + head * from.head + e0);
            if (a.rot && (is_k || is_q)) x = turned<L>(x, t, a, e0, c.bf);
            if (is_q) {
                if (live) *(uintx4*)(a.q_out + (token * a.q_heads + head) * c.d + e0) = x;
                continue;
            }
            uint16_t scale;
            const uint32_t ids = coded<L>(x, mid + ((is_k ? 0 : c.heads) + min(head, c.heads - 1)) * 16, c.bf, &scale);
            if (!live || !kept) continue;
            const int64_t row = (((slot >> c.page_shift) * c.heads + head) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
            *(uint32_t*)((is_k ? c.k_codes : c.v_codes) + row * (c.d / 2) + e0 / 2) = ids;
            if (e0 == 0) (is_k ? c.k_scale : c.v_scale)[row] = scale;
        }
    }
}

template <int L>
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
            const float s = lp_to_float((is_k ? c.k_scale : c.v_scale)[row], c.bf);
            const float* l = level + ((is_k ? 0 : c.heads) + head) * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = float_to_lp_any(l[(ids >> 8 * i) & 15] * s, c.bf);
                const uint32_t hi = float_to_lp_any(l[(ids >> (8 * i + 4)) & 15] * s, c.bf);
                r[i] = lo | (hi << 16);
            }
        }
        *(uintx4*)(out + (token * c.heads + head) * c.d + e0) = r;
    }
}

static int lanes_of(int d) { return d <= 32 ? 4 : d <= 64 ? 8 : d <= 128 ? 16 : 32; }

// Waves for all units, but no more workgroups than the chip holds at once: the rest is done in turns, so that the levels are loaded once.
static unsigned grid_for(int64_t units) {
    const int64_t blocks = cdiv(units, kAppendThreads / 64), most = (int64_t)device_cu_count() * 8;
    return (unsigned)(blocks < most ? blocks : most);
}

fk_status launch_kv_append(const KVView& c, const KVAppend& a, hipStream_t s) {
    const int L = lanes_of(c.d), rows = 64 / L;
    const int64_t groups = 2 * cdiv(c.heads, rows) + cdiv(a.q_heads, rows);
    const int per_unit = a.T * groups <= (int64_t)device_cu_count() * 32 ? 1 : (int)groups;
    const unsigned grid = grid_for(a.T * cdiv(groups, per_unit));
    const size_t lds = (size_t)c.heads * 16 * 2 * sizeof(float);
    if (L == 4) kv_append_kernel<4><<<grid, kAppendThreads, lds, s>>>(c, a, per_unit);
    else if (L == 8) kv_append_kernel<8><<<grid, kAppendThreads, lds, s>>>(c, a, per_unit);
    else if (L == 16) kv_append_kernel<16><<<grid, kAppendThreads, lds, s>>>(c, a, per_unit);
    else kv_append_kernel<32><<<grid, kAppendThreads, lds, s>>>(c, a, per_unit);
    FK_HIP(hipGetLastError());
    return FK_OK;
}

fk_status launch_kv_read(const KVView& c, const int64_t* slots, int64_t T, uint16_t* k_out, uint16_t* v_out, hipStream_t s) {
    const int L = lanes_of(c.d);
    const unsigned grid = grid_for(T * 2 * cdiv(c.heads, 64 / L));
    const size_t lds = (size_t)c.heads * 16 * 2 * sizeof(float);
    if (L == 4) kv_read_kernel<4><<<grid, kAppendThreads, lds, s>>>(c, slots, T, k_out, v_out);
    else if (L == 8) kv_read_kernel<8><<<grid, kAppendThreads, lds, s>>>(c, slots, T, k_out, v_out);
    else if (L == 16) kv_read_kernel<16><<<grid, kAppendThreads, lds, s>>>(c, slots, T, k_out, v_out);
    else kv_read_kernel<32><<<grid, kAppendThreads, lds, s>>>(c, slots, T, k_out, v_out);
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
