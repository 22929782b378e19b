// Attention over the 4-bit key/value cache: how a call is divided, and queries in a row.
#include "fk_kv_attend.h"

namespace fk {

KVPlan choose_kv_plan(const KVView& c, int q_heads, int B, int max_q, int64_t reach) {
    const int group = q_heads / c.heads, ND = c.d / 32;
    const int64_t rows = (int64_t)max_q * group, units = device_cu_count();
    KVPlan p;
    p.splits = 1;
    p.chunk = INT32_MAX / 2;
    // Waves with rows of their own need no exchange at the end, but the rows' workgroups alone have to fill the chip (8 x 5 queries of 16
    // heads of 256 over 4000 tokens: 16 workgroups 235 us, divided by tokens too 23); otherwise the tokens are divided.
    const int64_t own_blocks = (int64_t)B * c.heads * cdiv(rows, 16 * own_tiles(ND) * own_waves(own_tiles(ND)));
    if (rows > 16 * join_tiles(ND) && own_blocks >= units) {
        p.join = false;
        p.tiles = own_tiles(ND);
        p.row_blocks = (int)cdiv(rows, 16 * p.tiles);
        return p;
    }
    p.join = true;
    p.tiles = (int)std::min(cdiv(rows, 16), (int64_t)join_tiles(ND));
    p.row_blocks = (int)cdiv(rows, 16 * p.tiles);
    // One workgroup to a compute unit: 8 heads, one sequence of 131072 tokens 64 splits 38.2 us, 32 35.6, 24 41.4.
    const int64_t wg = kJoinWaves * kStep, blocks = (int64_t)B * c.heads * p.row_blocks;
    const int64_t want = blocks >= units ? 1 : units / blocks, steps = cdiv(reach, wg);
    // Splitting costs the second launch, about four steps of a workgroup: 8 heads of 128, one sequence of 700 tokens (3 steps) 10.1 us
    // in one piece and 10.0 in three, of 1500 (6) 13.8 and 10.4 in six; 24 sequences of 2048 (8), 4 heads of 64, 13.3 and 13.0 in two.
    p.splits = (int)std::min({want, steps, (int64_t)kMostSplits});
    if (steps - cdiv(steps, p.splits) <= 4) p.splits = 1;
    if (p.splits > 1) {
        p.chunk = cdiv(steps, p.splits) * wg;
        return p;
    }
    // Many short sequences: a tile to a wave, eight to a workgroup, saves the workgroups' fixed cost and gives up dividing the tokens.  In tenths of a
    // microsecond, fitted to 986 measured pairs from 32 to 256 channels, 1 to 4 tiles and 9 to 500 tokens (of which it takes the slower one where that
    // costs 0.6 % on average, and tiles where they are up to 2 % slower): workgroups that share their rows and hold at most 128 registers run in
    // pairs on a compute unit, others in rounds; each takes a time of its own and one a step of 256 tokens.  Tiles take theirs a step of 32.
    // One query of 4 heads to each of 8 heads of 128: 64 sequences of 100 tokens 10.3 us shared and 10.7 in tiles, of 32 9.5 and 6.6; 128 of 300
    // 23 and 18; of 256 channels 64 of 200 22.6 and 21.5, 32 of 200 12.4 and 21.2.
    const int64_t tiles = cdiv(rows, 16), own = cdiv(B * tiles, 8) * c.heads, more = std::max(blocks - units, (int64_t)0),
                  more_own = std::max(own - units, (int64_t)0), w = ND * p.tiles, own_steps = cdiv(reach, kStep);
    const bool pairs = w <= 2 || (p.tiles == 1 && ND <= 4);
    const int64_t shared_cost = pairs ? (40 + 5 * w + (4 + 3 * w) * steps) * units + (15 + w + (7 + 2 * w) * steps) * more
                                      : (60 + 2 * w + (10 + 2 * w) * steps) * cdiv(blocks, units) * units;
    const int64_t own_cost = (38 + 4 * ND + (7 + 2 * ND) * own_steps) * units + (15 + 9 * ND + (6 + 6 * ND) * own_steps) * more_own;
    if (own_cost < shared_cost) {
        p.join = false;
        p.tiles = 1;
        p.row_blocks = (int)tiles;
    }
    return p;
}

fk_status launch_kv_attend(const KVView& c, const KVAttend& a, const KVPlan& p, hipStream_t s) { return launch_attend<false>(c, a, p, s); }

}  // namespace fk
