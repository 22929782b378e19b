// Internal declarations of the 4-bit key/value cache (fk_kv_*.hip; not part of the ABI).
#pragma once

#include "fk_common.h"

namespace fk {

// round-to-nearest-even from fp32, infinities and NaN included
__device__ __forceinline__ uint16_t float_to_lp_any(float f, bool bf) {
    return bf ? __builtin_bit_cast(uint16_t, (__bf16)f) : __builtin_bit_cast(uint16_t, (_Float16)f);
}

// two of them in one register
template <bool BF>
__device__ __forceinline__ uint32_t pack_lp(float lo, float hi) {
    typedef float float2v __attribute__((ext_vector_type(2)));
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef _Float16 half2v __attribute__((ext_vector_type(2)));
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{lo, hi}, bf2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{lo, hi}, half2v));
}

// Rows of type t at element strides.
struct KVRows {
    const uint16_t* at;
    int64_t token, head;
};

// The cache as the kernels see it.
struct KVView {
    uint8_t *k_codes, *v_codes;
    uint16_t *k_scale, *v_scale;
    const uint16_t *k_levels, *v_levels;
    int64_t pages;
    int page_shift, heads, d;
    bool bf;
};

struct KVAppend {
    KVRows k, v, q;
    const int64_t* slots;
    int64_t T;
    const float* cos_sin;
    const int32_t* positions;
    int64_t max_pos;
    int rot, interleaved, q_heads;
    uint16_t* q_out;
};

struct KVAttend {
    KVRows q;
    int q_heads;
    int64_t Tq;
    const int32_t *pages, *lens, *q_start;
    int max_pages, B, max_q;
    float scale;
    int causal, window;
    uint16_t* out;
    float* lse;
    float* part;          // workspace: see kv_partial_floats
};

// Waves of a workgroup with rows of their own: four, two workgroups to a compute unit; with one tile each eight, that share one table.
constexpr int own_waves(int tiles) { return tiles == 1 ? 8 : 4; }

// How an attention call is divided.
struct KVPlan {
    int tiles;            // tiles of 16 query rows (query token, head of the group) in a wave
    bool join;            // the waves of a workgroup share the rows and divide the tokens; otherwise each has rows of its own
    int row_blocks;       // along the rows of a sequence and cache head: workgroups, or tiles of waves with rows of their own
    int splits;           // workgroups along the tokens
    int64_t chunk;        // tokens of a split, a multiple of what the waves of a workgroup take at a time
};
// `reach`: the most tokens that the queries of a sequence see together.  More of them never give fewer splits.
KVPlan choose_kv_plan(const KVView& c, int q_heads, int B, int max_q, int64_t reach);
// floats of one split's partial result: per query row its maximum and sum, and its d sums
inline int64_t kv_partial_floats(const KVPlan& p, int d) { return (int64_t)p.tiles * 16 * (d + 2); }
inline size_t kv_partial_bytes(const KVPlan& p, int d, int heads, int B) {
    return p.splits <= 1 ? 0 : (size_t)B * heads * p.row_blocks * p.splits * kv_partial_floats(p, d) * 4;
}

fk_status launch_kv_append(const KVView& c, const KVAppend& a, hipStream_t s);
fk_status launch_kv_read(const KVView& c, const int64_t* slots, int64_t T, uint16_t* k_out, uint16_t* v_out, hipStream_t s);
fk_status launch_kv_attend(const KVView& c, const KVAttend& a, const KVPlan& p, hipStream_t s);

}  // namespace fk
