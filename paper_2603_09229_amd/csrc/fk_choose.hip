// Which places of a sequence stay in the 4-bit key/value cache: its first ones, its last ones, and of the others those with the largest weights.
//
// Weights become 32-bit integers of the same order (NaN below all of them).  With m of the middle ones to be kept, the m-th largest value T is
// found 8 bits at a time, by counting how many of the values that share the bits found so far have which next ones; then those above T
// stay, and of those equal to T the first ones until there are m.  The places are written in ascending order by a prefix sum.
#include "fk_device.h"
#include "fk_evict.h"

namespace fk {

constexpr int kChooseThreads = 1024;

// order of weights as integers; 0 is NaN alone
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);                  // (-0 becomes 0)
    return w != w ? 0u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

__global__ __launch_bounds__(kChooseThreads) void kv_choose_kernel(KVView c, KVChoose a) {
    constexpr int WAVES = kChooseThreads / 64;
    __shared__ int bins[256];
    __shared__ int above[WAVES], equal[WAVES];
    __shared__ uint32_t found;
    __shared__ int missing;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    int32_t* kept = a.kept + ((int64_t)b * c.heads + h) * a.keep;
    if (h == 0 && tid == 0) a.counts[b] = min(len, a.keep);
    if (len <= a.keep) {
        for (int j = tid; j < a.keep; j += kChooseThreads) kept[j] = j < len ? j : -1;
        return;
    }
    const int32_t* table = a.pages + (int64_t)b * a.max_pages;
    auto value = [&](int t) {
        const int page = min(max(table[t >> c.page_shift], 0), (int)c.pages - 1);
        return order_of(a.mass[(((int64_t)page * c.heads + h) << c.page_shift) + (t & ((1 << c.page_shift) - 1))]);
    };
    const int from = a.first, to = len - a.last;
    if (tid == 0) {
        found = 0;
        missing = a.keep - a.first - a.last;
    }
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) bins[tid] = 0;
        __syncthreads();
        const uint32_t prefix = found;
        for (int t = from + tid; t < to; t += kChooseThreads) {
            const uint32_t v = value(t);
            if (shift == 24 || (v ^ prefix) >> (shift + 8) == 0) atomicAdd(&bins[v >> shift & 255], 1);
        }
        __syncthreads();
        if (wave == 0) {                                          // lane l: bins 255 - 4 l and the three below
            int own[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += own[i] = bins[255 - 4 * lane - i];
            int before = sum;
            for (int o = 1; o < 64; o *= 2) {
                const int x = __shfl_up(before, o);
                if (lane >= o) before += x;
            }
            before -= sum;
            const int want = missing;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < want && want <= before + own[i]) {
                    found = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
                    missing = want - before;
                }
                before += own[i];
            }
        }
        __syncthreads();
    }
    const uint32_t threshold = found;
    const int ties = missing, middle = a.keep - a.first - a.last;
    int done = 0, tied = 0;                                       // places written, ties met
    for (int t0 = 0; t0 < len; t0 += kChooseThreads) {
        const int t = t0 + tid;
        const bool inside = t >= from && t < to && middle > 0;
        const uint32_t v = inside ? value(t) : 0;
        const bool more = (t < len && (t < from || t >= to)) || (inside && v > threshold), tie = inside && v == threshold;
        const uint64_t mores = __ballot(more), same = __ballot(tie), lower = ((uint64_t)1 << lane) - 1;
        if (lane == 0) {
            above[wave] = __popcll(mores);
            equal[wave] = __popcll(same);
        }
        __syncthreads();
        int at = done, met = tied, all = 0, all_ties = 0;
        for (int w = 0; w < WAVES; ++w) {
            const int x = above[w], y = equal[w];
            at += w < wave ? x : 0;
            met += w < wave ? y : 0;
            all += x;
            all_ties += y;
        }
        // places before this one: those that stay for sure and the ties that still found room
        const int ties_before = met + __popcll(same & lower);
        const int place = at + __popcll(mores & lower) + min(ties_before, ties);
        if (more || (tie && ties_before < ties)) kept[place] = t;
        done += all;
        tied += all_ties;
        __syncthreads();
    }
}

fk_status launch_kv_choose(const KVView& c, const KVChoose& a, int64_t, hipStream_t s) {
    kv_choose_kernel<<<dim3(c.heads, a.B), kChooseThreads, 0, s>>>(c, a);
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
