// Rows of the 4-bit key/value cache moved to the front of their sequences.
//
// A wave moves the keys and the values (in place, one of them) of 64 rows of one sequence and head: a lane finds where a row is and where it
// goes, then the lanes take the rows' pieces of 16 bytes side by side, all of them on their way at once.  Into other pages that is all, and
// waves know nothing of each other.
//
// In place the places ascend, so that a row never goes behind where it was.  Rows that come from behind all places that are written
// (place >= count) are moved like those into other pages, after the others; of these one workgroup takes all in order, a tile at a time:
// into registers, a barrier, and out again.  A tile's rows are written over places that only this tile or an earlier one reads, so the next
// tile's places may be looked up before this one is written, and its rows read without another barrier.  Of n rows of a sequence of L
// that are spread evenly n^2 / L are moved in order.
//
// What bounds it: bytes.  32 sequences of up to 8192 tokens, 8 heads of 128, a quarter stays: 147 MB in 46 us, 3.2 TB/s (a copy of as many bytes 30;
// rows of 64 bytes at random use every other half of the 128 that memory gives, in a row they take 40).  In order: the way to memory and back of
// every tile.
#include "fk_device.h"
#include "fk_evict.h"

namespace fk {

constexpr int kCompactWaves = 4;         // of a workgroup where waves are on their own,
constexpr int kOrderedWaves = 16;        // and where it takes a sequence's rows in order
// Rows of a lane in a tile of long lists: what 128 registers hold
constexpr int ordered_rows(int ND) { return ND <= 2 ? 4 : ND <= 4 ? 2 : 1; }

enum { kAllRows, kNearRows, kFarRows };  // near: from places below `count`, far: from others

// SETS: rows of a lane in a tile
template <int ND, bool ORDERED, int SETS>
__global__ __launch_bounds__(64 * (ORDERED ? kOrderedWaves : kCompactWaves)) void kv_compact_kernel(KVView c, KVCompact a, int which) {
    constexpr int WAVES = ORDERED ? kOrderedWaves : kCompactWaves, TILE = 64 * WAVES * SETS;
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int count = min(max(a.counts[b], 0), a.max_kept);
    const int32_t* kept = a.kept + ((int64_t)b * a.kept_heads + (a.kept_heads > 1 ? h : 0)) * a.max_kept;
    const int64_t start = a.start ? a.start[b] : 0;
    // the cache's row of a place of the sequence, -1 outside
    auto row_of = [&](const int32_t* pages, int max_pages, int64_t place) -> int64_t {
        if (place < 0 || place >= (int64_t)max_pages << c.page_shift) return -1;
        const int64_t page = pages[(int64_t)b * max_pages + (place >> c.page_shift)];
        if (page < 0 || page >= c.pages) return -1;
        return ((page * c.heads + h) << c.page_shift) + (place & ((1 << c.page_shift) - 1));
    };
    // keys and values of a row: both, or in order, where there are few workgroups, one of them
    constexpr int SIDES = ORDERED ? 1 : 2;
    uintx4* codes[SIDES];
    uint16_t* scales[SIDES];
    bool masses = a.mass != nullptr;
    if constexpr (ORDERED) {
        const bool values = blockIdx.x;
        codes[0] = (uintx4*)(values ? c.v_codes : c.k_codes);
        scales[0] = values ? c.v_scale : c.k_scale;
        masses = masses && values;
    } else {
        codes[0] = (uintx4*)c.k_codes;
        codes[1] = (uintx4*)c.v_codes;
        scales[0] = c.k_scale;
        scales[1] = c.v_scale;
    }
    int64_t from[SETS], to[SETS];                                 // of the lane's rows; -1: none, or one that stays where it is
    auto look_up = [&](int64_t j0) {
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            const int64_t j = j0 + (s * WAVES + wave) * 64 + lane;
            from[s] = to[s] = -1;
            const int place = j < count ? kept[j] : -1;
            if (place < 0 || (which == kNearRows && place >= count) || (which == kFarRows && place < count)) continue;
            from[s] = row_of(a.pages, a.max_pages, start + place);
            to[s] = row_of(a.to_pages, a.to_max_pages, start + j);
            if (from[s] < 0 || to[s] < 0 || from[s] == to[s]) from[s] = to[s] = -1;
        }
    };
    const int first = ORDERED ? 0 : blockIdx.x * TILE;
    if (first >= count) return;
    look_up(first);
    for (int64_t j0 = first; j0 < (ORDERED ? count : min(count, first + TILE)); j0 += TILE) {
        if (which == kNearRows && kept[j0] >= count) break;       // and so are all behind it
        uintx4 piece[SETS][SIDES][ND];
        uint16_t scale[SETS][SIDES];
        float mass[SETS];
        int64_t target[SETS];
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
#pragma unroll
            for (int k = 0; k < ND; ++k) {
                const int64_t at = __shfl(from[s], (k * 64 + lane) / ND);
                if (at >= 0) {
#pragma unroll
                    for (int x = 0; x < SIDES; ++x) piece[s][x][k] = codes[x][at * ND + (k * 64 + lane) % ND];
                }
            }
            if (from[s] >= 0) {
#pragma unroll
                for (int x = 0; x < SIDES; ++x) scale[s][x] = scales[x][from[s]];
                if (masses) mass[s] = a.mass[from[s]];
            }
            target[s] = to[s];
        }
        if constexpr (ORDERED) {
            look_up(j0 + TILE);
            // every row of the tile is in registers before one of them is written
            __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        }
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
#pragma unroll
            for (int k = 0; k < ND; ++k) {
                const int64_t at = __shfl(target[s], (k * 64 + lane) / ND);
                if (at >= 0) {
#pragma unroll
                    for (int x = 0; x < SIDES; ++x) codes[x][at * ND + (k * 64 + lane) % ND] = piece[s][x][k];
                }
            }
            if (target[s] >= 0) {
#pragma unroll
                for (int x = 0; x < SIDES; ++x) scales[x][target[s]] = scale[s][x];
                if (masses) a.mass[target[s]] = mass[s];
            }
        }
    }
}

template <int ND>
static void launch_width(const KVView& c, const KVCompact& a, hipStream_t s) {
    const dim3 grid((unsigned)cdiv(a.max_kept, 64 * kCompactWaves), c.heads, a.B), ordered(2, c.heads, a.B);
    if (a.pages != a.to_pages) {
        kv_compact_kernel<ND, false, 1><<<grid, 64 * kCompactWaves, 0, s>>>(c, a, kAllRows);
    } else if (a.max_kept <= 4096 || 2 * (int64_t)a.B * c.heads >= device_cu_count()) {
        // Few tiles, or workgroups for the whole chip: a second launch gains nothing.  8 heads of 128: 8 sequences of 8192 cut down to 4096 18.5 us so
        // and 23.7 in two launches, 64 149 and 173; one of 65536 to 6000 18.8 and 11.3, to 29000 71 and 47, or to its last 29000 62 and 17.
        kv_compact_kernel<ND, true, 1><<<ordered, 64 * kOrderedWaves, 0, s>>>(c, a, kAllRows);
    } else {
        kv_compact_kernel<ND, true, ordered_rows(ND)><<<ordered, 64 * kOrderedWaves, 0, s>>>(c, a, kNearRows);
        kv_compact_kernel<ND, false, 1><<<grid, 64 * kCompactWaves, 0, s>>>(c, a, kFarRows);
    }
}

fk_status launch_kv_compact(const KVView& c, const KVCompact& a, hipStream_t s) {
    switch (c.d / 32) {
        case 1: launch_width<1>(c, a, s); break;
        case 2: launch_width<2>(c, a, s); break;
        case 3: launch_width<3>(c, a, s); break;
        case 4: launch_width<4>(c, a, s); break;
        case 5: launch_width<5>(c, a, s); break;
        case 6: launch_width<6>(c, a, s); break;
        case 7: launch_width<7>(c, a, s); break;
        default: launch_width<8>(c, a, s); break;
    }
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
