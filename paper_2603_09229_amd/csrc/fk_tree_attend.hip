// Attention of a tree of drafted tokens over the 4-bit key/value cache: the kernels of fk_kv_attend.h, with the tree's mask.
//
// The n queries of a sequence are its last n tokens, which are in the cache already.  All of them see what lies before the tree, which is
// where nearly all of the time goes and where nothing differs from queries in a row; of the tree's own n tokens they see those whose bits are set.  So the
// mask is only looked at in the steps of 32 tokens that reach past the prefix, two words a row and step, shifted to the step's first
// token; the bits of tokens before the tree count as set, so that a step may begin anywhere.
#include "fk_kv_attend.h"

namespace fk {

// As for queries in a row, but for the tiles of workgroups that share their rows and do not divide the tokens.  A tree has some dozen query
// tokens, more rows than one tile, and few sequences leave most of the chip idle: fewer tiles, and more workgroups that each decode the same codes.
// The cost, in tenths of a microsecond, is fitted to 21 sizes from 32 to 256 channels, 9 to 100 tokens a tree and 300 to 6000 before it, 1 to 4 tiles: a
// workgroup's first six steps of 256 tokens wait for memory more than later ones; those that hold at most 128 registers run in pairs on
// a compute unit, others in rounds.  One tree of 13 tokens, 8 heads of 128, 4 queries each, 700 tokens: three tiles 18.2 us, two 14.4, one 11.3; 8 of
// 60 over 1500: 53.5, 45.1, 47.4; 8 of 40, 8 heads of 64, over 6000: 43.1, 55.1, 58.6.
static KVPlan choose_tree_plan(const KVView& c, int q_heads, int B, int max_q, int64_t reach) {
    KVPlan p = choose_kv_plan(c, q_heads, B, max_q, reach);
    const int64_t rows = (int64_t)max_q * (q_heads / c.heads), ND = c.d / 32, units = device_cu_count(), steps = cdiv(reach, (int64_t)kJoinWaves * kStep);
    if (!p.join && p.tiles > 1 && p.tiles == join_tiles((int)ND)) {
        // Waves with rows of their own want two to a SIMD.  Trees often have fewer: then workgroups that share their rows are done sooner.  Both in tenths of a
        // microsecond: a wave's step of 32 tokens takes 11 w / 10 alone on its SIMD and 6 w / 10 as one of several; a workgroup's of 256 tokens 16 w / 10, and
        // rounds of them a time of their own.  16 trees of 60 tokens over 8000, 8 heads of 128, 4 queries each: 330 us with rows of their own,
        // 220 shared; 32 of 30, 8 heads of 64, over 6000: 197 and 97; of 200 over 3000, enough waves, 244 with rows of their own.
        const int64_t w = ND * p.tiles, waves = (int64_t)B * c.heads * cdiv(rows, 16 * p.tiles), each = cdiv(waves, 4 * units);
        const int64_t own = 40 + cdiv(reach, (int64_t)kStep) * (each == 1 ? 11 * w : 6 * w * each) / 10;
        const int64_t shared = cdiv(waves, units) * (80 + 5 * w + steps * 16 * w / 10);
        if (shared < own) p.join = true;
        return p;
    }
    if (!p.join || p.splits > 1) return p;
    int64_t least = INT64_MAX;
    for (int tiles = p.tiles; tiles >= 1; --tiles) {
        const int64_t blocks = (int64_t)B * c.heads * cdiv(rows, 16 * tiles), w = ND * tiles, early = std::min(steps, (int64_t)6), late = steps - early;
        int64_t cost = 0;
        if (w <= 2 || (tiles == 1 && ND <= 4) || (tiles == 2 && ND == 2)) {
            const int64_t more = std::max(blocks - units, (int64_t)0);
            cost = 50 + 6 * w + 16 * early + (6 + w) * late + (17 * w + (46 + 8 * w) * steps / 10) * (more + cdiv(more, units) * units) / (2 * units);
        } else {
            cost = (140 + 11 * w - 24 * (6 - early) + (35 + 12 * w) * late / 10) * cdiv(blocks, units);
        }
        if (cost < least) {
            least = cost;
            p.tiles = tiles;
            p.row_blocks = (int)cdiv(rows, 16 * tiles);
        }
    }
    return p;
}

// Ragged sequences: the longest first, where there are rounds of workgroups and these are long enough for the look at the lengths.  8 trees of 121 tokens over
// up to 20000 361 us in the order of the call, 346 so; 40 of 64 over up to 4096 (16 steps) 126 and 133.
static bool comes_longest_first(const KVView& c, const KVPlan& p, int B, int64_t reach, int window) {
    const int64_t blocks = (int64_t)B * c.heads * p.row_blocks, steps = cdiv(reach, (int64_t)kJoinWaves * kStep);
    return p.join && p.splits == 1 && !window && B > 1 && B <= 64 && blocks > device_cu_count() && steps >= 32;
}

}  // namespace fk

using namespace fk;

extern "C" int fk_kv_plan_tree(const fk_kv_cache* cache, int q_heads, int B, int max_q, int64_t max_len, int window, char* buf, size_t buf_bytes) {
    KVView c;
    FK_TRY(check_plan("fk_kv_plan_tree", cache, q_heads, B, max_q, max_len, window, buf, buf_bytes, &c));
    window = std::min(window, 1 << 30);
    const int64_t reach = reach_of(window, max_q + 1, max_len);
    const KVPlan p = choose_tree_plan(c, q_heads, B, max_q, reach);
    describe_plan(p, c, B, comes_longest_first(c, p, B, reach, window) ? ",longest_first" : "", buf, buf_bytes);
    return FK_OK;
}

extern "C" fk_status fk_kv_attend_tree(const fk_kv_cache* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_heads,
                                       int64_t Tq, const int32_t* pages, int max_pages, const int32_t* lens, const int32_t* q_start, int B,
                                       int max_q, int64_t max_len, float scale, int window, const uint64_t* tree, int words, void* out,
                                       float* lse, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "fk_kv_attend_tree";
    KVView c;
    fk_status why;
    if (!view_of(fn, cache, true, &c, &why)) return why;
    FK_TRY(check_queries(fn, c, q_heads, Tq, B, max_q, max_len));
    if (max_pages < 1 || window < 0 || (!q_start && Tq != (int64_t)B * max_q)) {
        set_error("%s: max_pages=%d, window=%d, or Tq=%lld without q_start is not B * max_q", fn, max_pages, window, (long long)Tq);
        return FK_EINVAL;
    }
    if (words < 1 || (int64_t)words * 64 < max_q) {
        set_error("%s: %d words of 64 bits for trees of up to %d tokens", fn, words, max_q);
        return FK_EINVAL;
    }
    if (!(fabsf(scale) <= 1e38f)) {                               // (times log2 e it has to be finite)
        set_error("%s: scale=%g is not a number up to 1e38", fn, (double)scale);
        return FK_EINVAL;
    }
    // (a row of the mask is found by 32 bits)
    if ((int64_t)max_pages << c.page_shift > (1 << 30) || Tq > (((int64_t)1 << 32) - 1) / 8 / words) {
        set_error("%s: unsupported size max_pages=%d of %d tokens, or a mask of %lld x %d words", fn, max_pages, 1 << c.page_shift,
                  (long long)Tq, words);
        return FK_EUNSUPPORTED;
    }
    if (max_len == 0) max_len = (int64_t)max_pages << c.page_shift;
    window = std::min(window, 1 << 30);
    if (Tq == 0) return FK_OK;
    FK_TRY(need(fn, "q", q, 2));
    FK_TRY(need(fn, "pages", pages, 4));
    FK_TRY(need(fn, "lens", lens, 4));
    if (q_start) FK_TRY(need(fn, "q_start", q_start, 4));
    FK_TRY(need(fn, "tree", tree, 8));
    FK_TRY(need(fn, "out", out, 16));
    if (lse) FK_TRY(need(fn, "lse", lse, 4));
    FK_TRY(need(fn, "ws", ws, 256));
    const int64_t reach = reach_of(window, max_q + 1, max_len);
    const KVPlan p = choose_tree_plan(c, q_heads, B, max_q, reach);
    const size_t bytes = kv_partial_bytes(p, c.d, c.heads, B);
    if (ws_bytes < bytes) {
        set_error("%s: workspace too small: %zu bytes given, %zu needed", fn, ws_bytes, bytes);
        return FK_EWORKSPACE;
    }
    const KVAttend a{{(const uint16_t*)q, q_token_stride, q_head_stride}, q_heads, Tq, pages, lens, q_start, max_pages, B, max_q,
                     scale, 0, window, (uint16_t*)out, lse, (float*)ws, tree, words};
    return launch_attend<true>(c, a, p, (hipStream_t)stream, comes_longest_first(c, p, B, reach, window));
}
