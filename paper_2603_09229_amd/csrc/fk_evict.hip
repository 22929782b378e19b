// C-ABI entry points that keep the 4-bit key/value cache small: argument checks and launches.
#include <math.h>

#include <algorithm>

#include "fk_evict.h"

using namespace fk;

// Page tables and lengths of B sequences.
static fk_status check_sequences(const char* fn, const KVView& c, int max_pages, int B) {
    if (max_pages < 1 || B < 1) {
        set_error("%s: max_pages=%d and B=%d must be positive", fn, max_pages, B);
        return FK_EINVAL;
    }
    if (B > 65535 || (int64_t)max_pages << c.page_shift > (1 << 30)) {
        set_error("%s: unsupported size B=%d max_pages=%d of %d tokens", fn, B, max_pages, 1 << c.page_shift);
        return FK_EUNSUPPORTED;
    }
    return FK_OK;
}

extern "C" {

fk_status fk_kv_weigh(const fk_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_heads, int64_t Tq,
                      const float* lse, const int32_t* pages, int max_pages, const int32_t* lens, const int32_t* q_start, int B, int max_q,
                      int64_t max_len, float scale, int causal, int window, const int32_t* known, float decay, const float* mass,
                      float* mass_out, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "fk_kv_weigh";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    FK_TRY(check_queries(fn, c, q_heads, Tq, B, max_q, max_len));
    if (window < 0 || (!q_start && Tq != (int64_t)B * max_q)) {
        set_error("%s: window=%d, or Tq=%lld without q_start is not B * max_q", fn, window, (long long)Tq);
        return FK_EINVAL;
    }
    if (!(fabsf(scale) <= 1e38f) || !(fabsf(decay) <= 3.402823466e38f)) {
        set_error("%s: scale=%g is not a number up to 1e38, or decay=%g is none", fn, (double)scale, (double)decay);
        return FK_EINVAL;
    }
    FK_TRY(check_sequences(fn, c, max_pages, B));
    if (max_len == 0) max_len = (int64_t)max_pages << c.page_shift;
    window = std::min(window, 1 << 30);
    if (Tq) {
        FK_TRY(need(fn, "q", q, 2));
        FK_TRY(need(fn, "lse", lse, 4));
    }
    FK_TRY(need(fn, "pages", pages, 4));
    FK_TRY(need(fn, "lens", lens, 4));
    if (q_start) FK_TRY(need(fn, "q_start", q_start, 4));
    if (known) FK_TRY(need(fn, "known", known, 4));
    FK_TRY(need(fn, "mass", mass, 4));
    FK_TRY(need(fn, "mass_out", mass_out, 4));
    const KVWeighPlan p = choose_weigh_plan(c, q_heads, B, max_q, std::min(max_len, (int64_t)max_pages << c.page_shift));
    const size_t bytes = weigh_workspace_bytes(p, c.heads, B);
    if (ws_bytes < bytes) {
        set_error("%s: workspace too small: %zu bytes given, %zu needed", fn, ws_bytes, bytes);
        return FK_EWORKSPACE;
    }
    if (bytes) FK_TRY(need(fn, "ws", ws, 256));
    const KVWeigh a{{(const uint16_t*)q, q_token_stride, q_head_stride}, q_heads, Tq, lse, pages, lens, q_start, max_pages, B, max_q, scale,
                    causal != 0, window, known, decay, mass, mass_out, (float*)ws};
    return launch_kv_weigh(c, a, p, (hipStream_t)stream);
}

size_t fk_kv_weigh_workspace_bytes(const fk_kv_cache* cache, int q_heads, int64_t Tq, int B, int max_q, int64_t max_len) {
    const char* fn = "fk_kv_weigh_workspace_bytes";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, false, &c, &why) || check_queries(fn, c, q_heads, Tq, B, max_q, max_len) != FK_OK) return 0;
    if (max_len < 1) {
        set_error("%s: max_len must be positive", fn);
        return 0;
    }
    return weigh_workspace_bytes(choose_weigh_plan(c, q_heads, B, max_q, max_len), c.heads, B);
}

fk_status fk_kv_choose(const fk_kv_cache* cache, const float* mass, const int32_t* pages, int max_pages, const int32_t* lens, int B,
                       int64_t max_len, int keep, int first, int last, int32_t* kept, int32_t* counts, void* ws,
                       size_t ws_bytes, void* stream) {
    const char* fn = "fk_kv_choose";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    FK_TRY(check_sequences(fn, c, max_pages, B));
    if (max_len < 0 || keep < 1 || first < 0 || last < 0 || (int64_t)first + last > keep) {
        set_error("%s: max_len=%lld is negative, or first=%d and last=%d are not within keep=%d", fn, (long long)max_len, first, last, keep);
        return FK_EINVAL;
    }
    if (keep > (1 << 30) || max_len > (1 << 30)) {
        set_error("%s: unsupported size keep=%d max_len=%lld", fn, keep, (long long)max_len);
        return FK_EUNSUPPORTED;
    }
    const int64_t room = (int64_t)max_pages << c.page_shift;
    FK_TRY(need(fn, "mass", mass, 4));
    FK_TRY(need(fn, "pages", pages, 4));
    FK_TRY(need(fn, "lens", lens, 4));
    FK_TRY(need(fn, "kept", kept, 4));
    FK_TRY(need(fn, "counts", counts, 4));
    if (counts < lens + B && lens < counts + B) {                 // (workgroups of all heads read lens, one of them writes counts)
        set_error("%s: counts overlaps lens", fn);
        return FK_EINVAL;
    }
    max_len = max_len ? std::min(max_len, room) : room;
    const size_t bytes = choose_workspace_bytes(c, B, max_len);
    if (ws_bytes < bytes) {
        set_error("%s: workspace too small: %zu bytes given, %zu needed", fn, ws_bytes, bytes);
        return FK_EWORKSPACE;
    }
    if (bytes) FK_TRY(need(fn, "ws", ws, 256));
    const KVChoose a{mass, pages, lens, max_pages, B, keep, first, last, kept, counts};
    return launch_kv_choose(c, a, max_len, ws, (hipStream_t)stream);
}

size_t fk_kv_choose_workspace_bytes(const fk_kv_cache* cache, int B, int64_t max_len) {
    const char* fn = "fk_kv_choose_workspace_bytes";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, false, &c, &why)) return 0;
    if (B < 1 || B > 65535 || max_len < 1 || max_len > (1 << 30)) {
        set_error("%s: B=%d is not in 1..65535 or max_len=%lld not in 1..2^30", fn, B, (long long)max_len);
        return 0;
    }
    return choose_workspace_bytes(c, B, max_len);
}

fk_status fk_kv_compact(const fk_kv_cache* cache, const int32_t* pages, int max_pages, const int32_t* kept, int kept_heads, int max_kept,
                        const int32_t* counts, const int32_t* start, const int32_t* to_pages, int to_max_pages, int B, float* mass,
                        void* stream) {
    const char* fn = "fk_kv_compact";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    FK_TRY(check_sequences(fn, c, max_pages, B));
    if (to_pages && to_pages != pages) FK_TRY(check_sequences(fn, c, to_max_pages, B));
    if (max_kept < 0 || (kept_heads != 1 && kept_heads != c.heads)) {
        set_error("%s: max_kept=%d is negative, or places for %d heads are neither for one nor for %d", fn, max_kept, kept_heads, c.heads);
        return FK_EINVAL;
    }
    if (max_kept > (1 << 30)) {
        set_error("%s: unsupported size max_kept=%d", fn, max_kept);
        return FK_EUNSUPPORTED;
    }
    if (max_kept == 0) return FK_OK;
    FK_TRY(need(fn, "pages", pages, 4));
    FK_TRY(need(fn, "kept", kept, 4));
    FK_TRY(need(fn, "counts", counts, 4));
    if (start) FK_TRY(need(fn, "start", start, 4));
    if (to_pages) FK_TRY(need(fn, "to_pages", to_pages, 4));
    if (mass) FK_TRY(need(fn, "mass", mass, 4));
    if (!to_pages || to_pages == pages) {
        to_pages = pages;
        to_max_pages = max_pages;
    }
    const KVCompact a{pages, to_pages, max_pages, to_max_pages, B, kept, counts, start, max_kept, kept_heads, mass};
    return launch_kv_compact(c, a, (hipStream_t)stream);
}

}  // extern "C"
