// Rows of the 4-bit key/value cache moved to the front of their sequences.
//
// A wave moves the keys and the values (in place, one of them) of 64 rows of one sequence and head: a lane finds where a row is and where it goes, then the lanes take the
// rows' pieces of 16 bytes side by side, all of them on their way at once.  Into other pages that is all, and waves know nothing of each
// other.  In place the places ascend, so that a row never goes behind where it was, and one workgroup takes all rows in order, a tile at
// a time: into registers, a barrier, and out again.  A tile's rows are written over places that only this tile or an earlier one reads.
// So the next tile's places may be looked up before this one is written, and its rows read without another barrier.
#include "fk_device.h"
#include "fk_evict.h"

namespace fk {

constexpr int kCompactWaves = 4;         // of a workgroup, into other pages,
constexpr int kCompactTile = 16;         // and in place: the rows of a tile in units of 64

template <int ND, bool IN_PLACE>
__global__ __launch_bounds__(64 * (IN_PLACE ? kCompactTile : kCompactWaves)) void kv_compact_kernel(KVView c, KVCompact a) {
    constexpr int WAVES = IN_PLACE ? kCompactTile : kCompactWaves, ROWS = 64 * WAVES;
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
    // keys and values of a row: both, or in place, where there are few workgroups, one of them
    constexpr int SIDES = IN_PLACE ? 1 : 2;
    uintx4* codes[SIDES];
    uint16_t* scales[SIDES];
    bool masses = a.mass != nullptr;
    if constexpr (IN_PLACE) {
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
    int64_t from = -1, to = -1;                                   // of the lane's row; -1: none, or one that stays where it is
    auto look_up = [&](int64_t j) {
        from = to = -1;
        const int place = j < count ? kept[j] : -1;
        if (place < 0) return;
        from = row_of(a.pages, a.max_pages, start + place);
        to = row_of(a.to_pages, a.to_max_pages, start + j);
        if (from < 0 || to < 0 || from == to) from = to = -1;
    };
    const int first = IN_PLACE ? 0 : blockIdx.x * ROWS;
    look_up((int64_t)first + wave * 64 + lane);
    for (int64_t j0 = first; j0 < (IN_PLACE ? count : min(count, first + ROWS)); j0 += ROWS) {
        uintx4 piece[SIDES][ND];
        uint16_t scale[SIDES];
        float mass = 0.f;
        int64_t target[ND];
#pragma unroll
        for (int k = 0; k < ND; ++k) {
            const int row = (k * 64 + lane) / ND, i = (k * 64 + lane) % ND;
            const int64_t at = __shfl(from, row);
            target[k] = __shfl(to, row);
            if (at >= 0) {
#pragma unroll
                for (int x = 0; x < SIDES; ++x) piece[x][k] = codes[x][at * ND + i];
            }
        }
        if (from >= 0) {
#pragma unroll
            for (int x = 0; x < SIDES; ++x) scale[x] = scales[x][from];
            if (masses) mass = a.mass[from];
        }
        const int64_t mine = to;
        if constexpr (IN_PLACE) {
            look_up(j0 + ROWS + wave * 64 + lane);
            // every row of the tile is in registers before one of them is written
            __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < ND; ++k)
            if (target[k] >= 0) {
#pragma unroll
                for (int x = 0; x < SIDES; ++x) codes[x][target[k] * ND + (k * 64 + lane) % ND] = piece[x][k];
            }
        if (mine >= 0) {
#pragma unroll
            for (int x = 0; x < SIDES; ++x) scales[x][mine] = scale[x];
            if (masses) a.mass[mine] = mass;
        }
    }
}

template <int ND>
static void launch_width(const KVView& c, const KVCompact& a, hipStream_t s) {
    if (a.pages == a.to_pages) {
        kv_compact_kernel<ND, true><<<dim3(2, c.heads, a.B), 64 * kCompactTile, 0, s>>>(c, a);
    } else {
        const dim3 grid((unsigned)cdiv(a.max_kept, 64 * kCompactWaves), c.heads, a.B);
        kv_compact_kernel<ND, false><<<grid, 64 * kCompactWaves, 0, s>>>(c, a);
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
