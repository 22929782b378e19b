// Internal declarations of what keeps a 4-bit key/value cache small: attention weights, choice of places, compaction (not part of the ABI).
#pragma once

#include "fk_kv.h"

namespace fk {

struct KVWeigh {
    KVRows q;
    int q_heads;
    int64_t Tq;
    const float* lse;
    const int32_t *pages, *lens, *q_start;
    int max_pages, B, max_q;
    float scale;
    int causal, window;
    const int32_t* known;
    float decay;
    const float* mass;
    float* out;
    float* part;          // workspace: sums of divided rows, [B * heads][splits][tokens]
};

struct KVChoose {
    const float* mass;
    const int32_t *pages, *lens;
    int max_pages, B, keep, first, last;
    int32_t *kept, *counts;
};

struct KVCompact {
    const int32_t *pages, *to_pages;
    int max_pages, to_max_pages, B;
    const int32_t *kept, *counts, *start;
    int max_kept, kept_heads;
    float* mass;
};

// How a call that weighs is divided.
struct KVWeighPlan {
    bool stream;          // more query rows than a workgroup keeps
    int row_waves;        // waves of a workgroup that share its tokens and divide the query rows
    int64_t chunk;        // tokens of a workgroup
    int blocks;           // workgroups along the tokens
    int splits;           // and along the query rows
};
inline size_t weigh_workspace_bytes(const KVWeighPlan& p, int heads, int B) {
    return p.splits <= 1 ? 0 : align_up((size_t)B * heads * p.splits * p.blocks * p.chunk * sizeof(float), 256);
}
KVWeighPlan choose_weigh_plan(const KVView& c, int q_heads, int B, int max_q, int64_t max_len);

fk_status launch_kv_weigh(const KVView& c, const KVWeigh& a, const KVWeighPlan& p, hipStream_t s);
size_t choose_workspace_bytes(const KVView& c, int B, int64_t max_len);
fk_status launch_kv_choose(const KVView& c, const KVChoose& a, int64_t max_len, void* ws, hipStream_t s);
fk_status launch_kv_compact(const KVView& c, const KVCompact& a, hipStream_t s);

}  // namespace fk
