// Rows of the 4-bit key/value cache moved to the front of their sequences.
//
// A workgroup moves keys or values of one sequence and head, a tile of rows at a time: where its rows are and go, all their codes and
// scales into registers, a barrier, and out again.  In place the places ascend, so that a row never goes behind where it was, and one
// workgroup takes all tiles in order: a tile's rows are written over places that only this tile or an earlier one reads.  Into
// other pages every tile has a workgroup of its own.
#include "fk_device.h"
#include "fk_evict.h"

namespace fk {

constexpr int kCompactThreads = 512;
constexpr int kCompactRows = 512;        // of a tile

template <int ND>
__global__ __launch_bounds__(kCompactThreads) void kv_compact_kernel(KVView c, KVCompact a, int in_place) {
    __shared__ int64_t source[kCompactRows], target[kCompactRows];
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
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
    uintx4* codes = (uintx4*)(values ? c.v_codes : c.k_codes);
    uint16_t* scales = values ? c.v_scale : c.k_scale;
    const int first = (blockIdx.x >> 1) * kCompactRows, all = in_place ? count : min(count, first + kCompactRows);
    for (int j0 = first; j0 < all; j0 += kCompactRows) {
        const int rows = min(kCompactRows, all - j0);
        int64_t from = -1, to = -1;
        if (tid < rows) {
            const int place = kept[j0 + tid];
            if (place >= 0) {
                from = row_of(a.pages, a.max_pages, start + place);
                to = row_of(a.to_pages, a.to_max_pages, start + j0 + tid);
                if (from < 0 || to < 0 || from == to) from = to = -1;
            }
        }
        source[tid] = from;
        target[tid] = to;
        __syncthreads();
        uintx4 piece[ND];
#pragma unroll
        for (int k = 0; k < ND; ++k) {
            const int i = k * kCompactThreads + tid, r = i / ND;
            const int64_t at = source[r];
            if (at >= 0) piece[k] = codes[at * ND + i % ND];
        }
        uint16_t scale = 0;
        float mass = 0.f;
        if (from >= 0) {
            scale = scales[from];
            if (values && a.mass) mass = a.mass[from];
        }
        // every row of the tile is in registers before one of them is written
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ND; ++k) {
            const int i = k * kCompactThreads + tid, r = i / ND;
            const int64_t at = target[r];
            if (at >= 0) codes[at * ND + i % ND] = piece[k];
        }
        if (from >= 0) {
            scales[to] = scale;
            if (values && a.mass) a.mass[to] = mass;
        }
        __syncthreads();
    }
}

fk_status launch_kv_compact(const KVView& c, const KVCompact& a, hipStream_t s) {
    const int in_place = a.pages == a.to_pages;
    const dim3 grid(2 * (in_place ? 1 : (unsigned)cdiv(a.max_kept, kCompactRows)), c.heads, a.B);
    switch (c.d / 32) {
        case 1: kv_compact_kernel<1><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        case 2: kv_compact_kernel<2><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        case 3: kv_compact_kernel<3><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        case 4: kv_compact_kernel<4><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        case 5: kv_compact_kernel<5><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        case 6: kv_compact_kernel<6><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        case 7: kv_compact_kernel<7><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
        default: kv_compact_kernel<8><<<grid, kCompactThreads, 0, s>>>(c, a, in_place); break;
    }
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
