// C-ABI entry points of the 4-bit key/value cache: argument checks and launches.
#include <math.h>
#include <stdio.h>

#include <algorithm>

#include "fk_kv.h"

namespace fk {

bool view_of(const char* fn, const fk_kv_cache* c, bool pointers, KVView* v, fk_status* why) {
    *why = FK_EINVAL;
    if (!c) {
        set_error("%s: the cache is NULL", fn);
        return false;
    }
    if (c->t != FK_F32 && c->t != FK_F16 && c->t != FK_BF16) {
        set_error("%s: unknown dtype %d", fn, (int)c->t);
        return false;
    }
    if (c->pages < 1 || c->page_size < 1 || c->heads < 1 || c->d < 1) {
        set_error("%s: pages, page_size, heads, d must be positive (%lld, %d, %d, %d)", fn, (long long)c->pages, c->page_size,
                  c->heads, c->d);
        return false;
    }
    if (c->t == FK_F32 || c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) || c->d % 32 ||
        c->d > 256 || c->heads > 256 || c->pages > INT32_MAX || c->pages > ((int64_t)1 << 40) / c->page_size) {
        set_error("%s: unsupported cache: page_size=%d heads=%d d=%d dtype=%d (need fp16 or bf16, a power of two from 16 to 65536, "
                  "at most 256 heads, d a multiple of 32 up to 256)", fn, c->page_size, c->heads, c->d, (int)c->t);
        *why = FK_EUNSUPPORTED;
        return false;
    }
    if (pointers) {
        const void* p[] = {c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->k_levels, c->v_levels};
        const char* name[] = {"k_codes", "v_codes", "k_scale", "v_scale", "k_levels", "v_levels"};
        for (int i = 0; i < 6; ++i)
            if (!p[i] || ((uintptr_t)p[i] & 15u)) {
                set_error("%s: %s is NULL or not 16-byte aligned", fn, name[i]);
                return false;
            }
    }
    *v = KVView{(uint8_t*)c->k_codes, (uint8_t*)c->v_codes, (uint16_t*)c->k_scale, (uint16_t*)c->v_scale,
                (const uint16_t*)c->k_levels, (const uint16_t*)c->v_levels, c->pages, __builtin_ctz((unsigned)c->page_size),
                c->heads, c->d, c->t == FK_BF16};
    *why = FK_OK;
    return true;
}

fk_status need(const char* fn, const char* name, const void* p, size_t to) {
    if (p && !((uintptr_t)p & (to - 1))) return FK_OK;
    set_error("%s: %s is NULL or not %zu-byte aligned", fn, name, to);
    return FK_EINVAL;
}

fk_status check_queries(const char* fn, const KVView& c, int q_heads, int64_t Tq, int B, int max_q, int64_t max_len) {
    if (q_heads < 1 || B < 1 || max_q < 1 || Tq < 0 || max_len < 0) {
        set_error("%s: q_heads, B, max_q must be positive, Tq and max_len not negative (%d, %d, %d, %lld, %lld)", fn, q_heads, B,
                  max_q, (long long)Tq, (long long)max_len);
        return FK_EINVAL;
    }
    if (q_heads % c.heads) {
        set_error("%s: %d query heads are no multiple of %d cache heads", fn, q_heads, c.heads);
        return FK_EINVAL;
    }
    if (B > 65535 || Tq > INT32_MAX || (int64_t)max_q * (q_heads / c.heads) > (1 << 30) || max_len > (1 << 30)) {
        set_error("%s: unsupported size B=%d Tq=%lld max_q=%d max_len=%lld", fn, B, (long long)Tq, max_q, (long long)max_len);
        return FK_EUNSUPPORTED;
    }
    return FK_OK;
}

int64_t reach_of(int window, int max_q, int64_t max_len) {
    return window ? std::min((int64_t)window + max_q - 1, max_len) : max_len;
}

fk_status check_plan(const char* fn, const fk_kv_cache* cache, int q_heads, int B, int max_q, int64_t max_len, int window, char* buf, size_t buf_bytes,
                     KVView* c) {
    if (!buf || buf_bytes == 0) {
        set_error("%s: no buffer", fn);
        return FK_EINVAL;
    }
    snprintf(buf, buf_bytes, "unsupported");
    fk_status why;
    if (!view_of(fn, cache, false, c, &why)) return why;
    FK_TRY(check_queries(fn, *c, q_heads, 0, B, max_q, max_len));
    if (max_len < 1 || window < 0) {
        set_error("%s: max_len=%lld is not positive or window=%d is negative", fn, (long long)max_len, window);
        return FK_EINVAL;
    }
    return FK_OK;
}

void describe_plan(const KVPlan& p, const KVView& c, int B, const char* more, char* buf, size_t buf_bytes) {
    const size_t bytes = align_up(kv_partial_bytes(p, c.d, c.heads, B), 256) + 256;
    if (p.join)
        snprintf(buf, buf_bytes, "rows_shared(tiles=%d,row_blocks=%d,splits=%d,chunk=%lld%s) workspace=%zu", p.tiles, p.row_blocks, p.splits,
                 (long long)(p.splits > 1 ? p.chunk : 0), more, bytes);
    else
        snprintf(buf, buf_bytes, "rows_own(tiles=%d,row_blocks=%d,waves=%d%s) workspace=%zu", p.tiles, p.row_blocks, own_waves(p.tiles),
                 p.row_blocks < own_waves(p.tiles) ? ",packed" : "", bytes);
}

}  // namespace fk

using namespace fk;

extern "C" {

fk_status fk_kv_append(const fk_kv_cache* cache, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                       const void* v, int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots, int64_t T,
                       const float* cos_sin, const int32_t* positions, int64_t max_pos, int rot, int interleaved,
                       const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_heads, void* q_out,
                       void* stream) {
    const char* fn = "fk_kv_append";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    if (T < 0 || rot < 0 || rot > c.d) {
        set_error("%s: T=%lld is negative or rot=%d is not in 0..%d", fn, (long long)T, rot, c.d);
        return FK_EINVAL;
    }
    if (rot % 16) {
        set_error("%s: rot=%d is no multiple of 16", fn, rot);
        return FK_EUNSUPPORTED;
    }
    if (T > INT32_MAX || q_heads > 65536) {
        set_error("%s: unsupported size T=%lld q_heads=%d", fn, (long long)T, q_heads);
        return FK_EUNSUPPORTED;
    }
    if ((q == nullptr) != (q_out == nullptr) || (q && q_heads < 1)) {
        set_error("%s: q, q_out and q_heads come together", fn);
        return FK_EINVAL;
    }
    if (T == 0) return FK_OK;
    FK_TRY(need(fn, "k", k, 2));
    FK_TRY(need(fn, "v", v, 2));
    FK_TRY(need(fn, "slots", slots, 8));
    if (q) {
        FK_TRY(need(fn, "q", q, 2));
        FK_TRY(need(fn, "q_out", q_out, 16));
    }
    if (rot) {
        FK_TRY(need(fn, "cos_sin", cos_sin, 16));
        FK_TRY(need(fn, "positions", positions, 4));
        if (max_pos < 1 || max_pos > INT32_MAX) {
            set_error("%s: max_pos=%lld is not in 1..2^31-1", fn, (long long)max_pos);
            return FK_EINVAL;
        }
    }
    const KVAppend a{{(const uint16_t*)k, k_token_stride, k_head_stride}, {(const uint16_t*)v, v_token_stride, v_head_stride},
                     {(const uint16_t*)q, q_token_stride, q_head_stride}, slots, T, cos_sin, positions, max_pos, rot,
                     interleaved != 0, q ? q_heads : 0, (uint16_t*)q_out};
    return launch_kv_append(c, a, (hipStream_t)stream);
}

fk_status fk_kv_read(const fk_kv_cache* cache, const int64_t* slots, int64_t T, void* k_out, void* v_out, void* stream) {
    const char* fn = "fk_kv_read";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    if (T < 0) {
        set_error("%s: T=%lld is negative", fn, (long long)T);
        return FK_EINVAL;
    }
    if (T > INT32_MAX) {
        set_error("%s: unsupported size T=%lld", fn, (long long)T);
        return FK_EUNSUPPORTED;
    }
    if (T == 0 || (!k_out && !v_out)) return FK_OK;
    FK_TRY(need(fn, "slots", slots, 8));
    if (k_out) FK_TRY(need(fn, "k_out", k_out, 16));
    if (v_out) FK_TRY(need(fn, "v_out", v_out, 16));
    return launch_kv_read(c, slots, T, (uint16_t*)k_out, (uint16_t*)v_out, (hipStream_t)stream);
}

size_t fk_kv_workspace_bytes(const fk_kv_cache* cache, int q_heads, int64_t Tq, int B, int max_q, int64_t max_len) {
    const char* fn = "fk_kv_workspace_bytes";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, false, &c, &why) || check_queries(fn, c, q_heads, Tq, B, max_q, max_len) != FK_OK) return 0;
    if (max_len < 1) {
        set_error("%s: max_len must be positive", fn);
        return 0;
    }
    const size_t n = kv_partial_bytes(choose_kv_plan(c, q_heads, B, max_q, max_len), c.d, c.heads, B);
    return align_up(n, 256) + 256;
}

int fk_kv_plan(const fk_kv_cache* cache, int q_heads, int B, int max_q, int64_t max_len, int window, char* buf, size_t buf_bytes) {
    KVView c;
    FK_TRY(check_plan("fk_kv_plan", cache, q_heads, B, max_q, max_len, window, buf, buf_bytes, &c));
    describe_plan(choose_kv_plan(c, q_heads, B, max_q, reach_of(window, max_q, max_len)), c, B, "", buf, buf_bytes);
    return FK_OK;
}

fk_status fk_kv_attend(const fk_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                       int q_heads, int64_t Tq, const int32_t* pages, int max_pages, const int32_t* lens,
                       const int32_t* q_start, int B, int max_q, int64_t max_len, float scale, int causal, int window,
                       void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "fk_kv_attend";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    FK_TRY(check_queries(fn, c, q_heads, Tq, B, max_q, max_len));
    if (max_pages < 1 || window < 0 || (!q_start && Tq != (int64_t)B * max_q)) {
        set_error("%s: max_pages=%d, window=%d, or Tq=%lld without q_start is not B * max_q", fn, max_pages, window, (long long)Tq);
        return FK_EINVAL;
    }
    if (!(fabsf(scale) <= 1e38f)) {                               // (times log2 e it has to be finite)
        set_error("%s: scale=%g is not a number up to 1e38", fn, (double)scale);
        return FK_EINVAL;
    }
    if ((int64_t)max_pages << c.page_shift > (1 << 30)) {
        set_error("%s: unsupported size max_pages=%d of %d tokens", fn, max_pages, 1 << c.page_shift);
        return FK_EUNSUPPORTED;
    }
    if (max_len == 0) max_len = (int64_t)max_pages << c.page_shift;
    // No two positions are further apart: positions are from -2^30 (max_q) to 2^30, and 32 bits hold one of them less the window.
    window = std::min(window, 1 << 30);
    if (Tq == 0) return FK_OK;
    FK_TRY(need(fn, "q", q, 2));
    FK_TRY(need(fn, "pages", pages, 4));
    FK_TRY(need(fn, "lens", lens, 4));
    if (q_start) FK_TRY(need(fn, "q_start", q_start, 4));
    FK_TRY(need(fn, "out", out, 16));
    if (lse) FK_TRY(need(fn, "lse", lse, 4));
    FK_TRY(need(fn, "ws", ws, 256));
    const KVPlan p = choose_kv_plan(c, q_heads, B, max_q, reach_of(window, max_q, max_len));
    const size_t bytes = kv_partial_bytes(p, c.d, c.heads, B);
    if (ws_bytes < bytes) {
        set_error("%s: workspace too small: %zu bytes given, %zu needed", fn, ws_bytes, bytes);
        return FK_EWORKSPACE;
    }
    const KVAttend a{{(const uint16_t*)q, q_token_stride, q_head_stride}, q_heads, Tq, pages, lens, q_start, max_pages, B, max_q,
                     scale, causal != 0, window, (uint16_t*)out, lse, (float*)ws};
    return launch_kv_attend(c, a, p, (hipStream_t)stream);
}

}  // extern "C"
