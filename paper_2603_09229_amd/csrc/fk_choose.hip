// Which places of a sequence stay in the 4-bit key/value cache: its first ones, its last ones, and of the others those with the largest weights.
//
// Weights become 32-bit integers of the same order (NaN below all of them).  With m of the middle ones to be kept, the m-th largest value T is
// found 11, 11 and 10 bits at a time, by counting how many of the values that share the bits found so far have which next ones; then
// those above T stay, and of those equal to T the first ones until there are m.  The places are written in ascending order by a prefix
// sum.  Nothing depends on the order in which the counts are added.
//
// A workgroup holds the weights of a sequence and head in registers, read once.  Sequences of more than kWhole tokens are divided among
// workgroups, and the four steps are launches of their own: each counts its part, the next one adds the parts' counts up.
//
// What bounds it.  One short sequence: latency, of the page and the weight behind each other, of three rounds of counting with three barriers each, and
// of the places' prefix sums.  A batch: about 550 vector instructions a wave, issued in 58 % of the cycles, and additions in LDS that meet in a
// bank, 46 % of its time: the leading 11 bits are sign, exponent and two bits of mantissa, and most weights fall into few of them.  In parts: four
// launches behind each other, and in the last three every workgroup adds all parts' counts up for the bin that all of them find.  8 heads: one sequence of 1100
// tokens 6.5 us, 64 of up to 8192 13.9 (15 MB, 1.1 TB/s; counted one weight a thread at a time from memory 29), one of 131072 in 16 parts 23.8 (in
// one workgroup 299).  Counts are held four times, so that lanes with the same leading bits wait less for each other.  Sums within a wave go by DPP,
// six instructions instead of six trips through LDS.
#include <algorithm>

#include "fk_device.h"
#include "fk_evict.h"

namespace fk {

constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
// Most tokens that one workgroup holds in registers.  8 heads of one sequence: 9000 tokens 13.7 us (five of 16 a thread's registers go through scratch
// memory: the bound of 64 lets workgroups run in pairs); 32 a thread no longer fit, 32000 tokens 54, and 33000 in parts 22.
constexpr int kWhole = 16 * kChooseThreads;
constexpr int kPart = 8 * kChooseThreads;     // fewest of a part
constexpr int kMostParts = 64;
constexpr int kBins = 2048;
constexpr int kCopies = 4;               // of the counts, so that lanes with the same bits meet less often

// A part's own place in the search, kept from launch to launch: bits found, how many with them are wanted, and how many places that stay lie in
// earlier parts.
struct ChooseState {
    uint32_t found;
    int missing, before;
};

struct ChooseArgs {
    KVView c;
    KVChoose a;
    int parts;
    int* counts;               // [2][B * heads][parts][kBins]
    ChooseState* state;        // [B * heads][parts]
};

// Order of weights as integers.  NaN is 1, below all of them; kNothing is behind the sequence's end and kProtected a place that stays in any
// case: both are bit patterns of NaN, which no weight's order is.  So nothing but the order decides: the `keep` largest stay.
constexpr uint32_t kNothing = 0, kProtected = 0xffffffffu;
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);                  // (-0 becomes 0)
    return w != w ? 1u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// Inclusive sum over the lanes of a wave, without a trip through LDS.
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // within rows of 16: from 1, 2, 4 and 8 lanes below
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // the sums of rows 0 and 2 to the rows above them
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // and of the lower half to the upper one
    return x;
}
// How many of the lanes below this one are in the mask.
__device__ __forceinline__ int lower_lanes(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

struct ChooseShared {
    __align__(16) int bins[kBins][kCopies];
    int waves[kChooseWaves], ties[kChooseWaves];
    ChooseState next;
    int ties_before;
};

// sums of the waves below this one and of all, from one number a wave
__device__ __forceinline__ int waves_below(const int* waves, int wave, int lane, int* all) {
    const int scan = wave_scan(lane < kChooseWaves ? waves[lane] : 0);
    *all = __builtin_amdgcn_readlane(scan, kChooseWaves - 1);
    return wave ? __builtin_amdgcn_readlane(scan, wave - 1) : 0;
}

// The bits of the wanted value and what is still wanted below it, from a thread's two counts in descending order; `earlier`: the same counts
// in earlier parts.
__device__ __forceinline__ void find_bin(ChooseShared& S, ChooseState& s, const int (&own)[2], const int (&earlier)[2], int shift, int tid, int* ties_before) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), sum = own[0] + own[1], scan = wave_scan(sum);
    if (lane == 63) S.waves[wave] = scan;
    __syncthreads();
    int all;
    const int below = waves_below(S.waves, wave, lane, &all), above = below + scan - sum;
    const int hit = above < s.missing && s.missing <= above + own[0] ? 0 : above + own[0] < s.missing && s.missing <= above + sum ? 1 : -1;
    if (hit >= 0) {                                               // one thread
        S.next.found = s.found | (uint32_t)(kBins - 1 - 2 * tid - hit) << shift;
        S.next.missing = s.missing - above - (hit ? own[0] : 0);
        S.ties_before = earlier[hit];
    }
    __syncthreads();
    s.found = S.next.found;
    s.missing = S.next.missing;
    *ties_before = S.ties_before;
}

// STAGE -1: everything; 0 to 3: one of four launches over parts.  A wave's tokens follow each other, 64 to an item.
template <int ITEMS, int STAGE>
__global__ __launch_bounds__(kChooseThreads, 8) void kv_choose_kernel(ChooseArgs A) {
    __shared__ ChooseShared S;
    const KVChoose& a = A.a;
    const KVView& c = A.c;
    const int h = blockIdx.x, b = blockIdx.y, part = STAGE < 0 ? 0 : blockIdx.z, parts = STAGE < 0 ? 1 : A.parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    int32_t* kept = a.kept + ((int64_t)b * c.heads + h) * a.keep;
    if (STAGE <= 0 && h == 0 && part == 0 && tid == 0) a.counts[b] = min(len, a.keep);
    if (len <= a.keep) {
        if (STAGE <= 0)
            for (int64_t j = (int64_t)part * kChooseThreads + tid; j < a.keep; j += (int64_t)parts * kChooseThreads) kept[j] = j < len ? (int)j : -1;
        return;
    }
    const int32_t* table = a.pages + (int64_t)b * a.max_pages;
    const int each = ((len + parts - 1) / parts + kChooseThreads - 1) / kChooseThreads * kChooseThreads;
    const int begin = (int)min((int64_t)part * each, (int64_t)len), end = (int)min((int64_t)begin + each, (int64_t)len);
    const int rounds = (end - begin + ITEMS * kChooseThreads - 1) / (ITEMS * kChooseThreads);

    uint32_t v[ITEMS];
    auto first_of = [&](int round) { return begin + (round * kChooseWaves + wave) * (ITEMS * 64) + lane; };
    auto load = [&](int round) {
        const int t0 = first_of(round);
        int page[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) page[i] = table[min(t0 + i * 64, len - 1) >> c.page_shift];
        float w[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int t = min(t0 + i * 64, len - 1), p = min(max(page[i], 0), (int)c.pages - 1);
            w[i] = a.mass[(((int64_t)p * c.heads + h) << c.page_shift) + (t & ((1 << c.page_shift) - 1))];
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int t = t0 + i * 64;
            v[i] = t >= end ? kNothing : t < a.first || t >= len - a.last ? kProtected : order_of(w[i]);
        }
    };
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < kBins * kCopies / 4 / kChooseThreads; ++i) ((uintx4*)S.bins)[i * kChooseThreads + tid] = uintx4{0, 0, 0, 0};
    };
    // (the counts are cleared: by `clear`, or by who read them last)
    auto count = [&](const ChooseState& s, int shift, int bits) {
        for (int r = 0; r < rounds; ++r) {
            if (rounds > 1) load(r);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (shift == 21 || (v[i] ^ s.found) >> (shift + bits) == 0)
                    atomicAdd(&S.bins[v[i] >> shift & ((1 << bits) - 1)][lane & (kCopies - 1)], 1);
        }
        __syncthreads();
    };
    // a thread's two counts, of bits 2047 - 2 tid and one less
    auto counted = [&](int (&own)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uintx4& at = *(uintx4*)S.bins[kBins - 1 - 2 * tid - i];
            const uintx4 x = at;
            if (STAGE < 0) at = uintx4{0, 0, 0, 0};
            own[i] = (int)(x[0] + x[1] + x[2] + x[3]);
        }
    };

    constexpr int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
    ChooseState s{0, a.keep, 0};
    int ties_before = 0;
    if (rounds == 1) load(0);                                     // (on its way while counts are cleared or added up)
    if constexpr (STAGE < 3) clear();
    if constexpr (STAGE < 0) {
        const int none[2] = {0, 0};
        __syncthreads();
        auto pass = [&](int shift, int bits) {
            count(s, shift, bits);
            int own[2];
            counted(own);
            find_bin(S, s, own, none, shift, tid, &ties_before);
        };
        pass(shifts[0], widths[0]);
#pragma unroll 1
        for (int p = 1; p < 3; ++p) pass(p == 1 ? shifts[1] : shifts[2], p == 1 ? widths[1] : widths[2]);
    } else {
        typedef int intx2 __attribute__((ext_vector_type(2)));
        const int64_t unit = (int64_t)b * c.heads + h, stage_ints = (int64_t)a.B * c.heads * parts * kBins;
        ChooseState* mine = A.state + unit * parts + part;
        if constexpr (STAGE > 0) {
            if (STAGE > 1) s = *mine;
            const int* all = A.counts + ((STAGE - 1) & 1) * stage_ints + unit * parts * kBins + (kBins - 2 - 2 * tid);
            int own[2] = {0, 0}, earlier[2] = {0, 0};
#pragma unroll 8
            for (int p = 0; p < parts; ++p) {
                const intx2 x = *(const intx2*)(all + (int64_t)p * kBins);
                own[0] += x[1];
                own[1] += x[0];
                earlier[0] += p < part ? x[1] : 0;
                earlier[1] += p < part ? x[0] : 0;
            }
            find_bin(S, s, own, earlier, shifts[STAGE - 1], tid, &ties_before);
            // places that stay in earlier parts: those above the bits found
            const uint32_t bin = (s.found >> shifts[STAGE - 1]) & ((1u << widths[STAGE - 1]) - 1), bin0 = kBins - 1 - 2 * tid;
            const int above = wave_scan((bin0 > bin ? earlier[0] : 0) + (bin0 > bin + 1 ? earlier[1] : 0));
            if (lane == 63) S.ties[wave] = above;
            __syncthreads();
            int sum;
            waves_below(S.ties, wave, lane, &sum);
            s.before += sum;
        }
        if constexpr (STAGE < 3) {
            __syncthreads();                                      // (cleared)
            count(s, shifts[STAGE], widths[STAGE]);
            int own[2];
            counted(own);
            *(intx2*)(A.counts + (STAGE & 1) * stage_ints + (unit * parts + part) * kBins + (kBins - 2 - 2 * tid)) = intx2{own[1], own[0]};
            if (STAGE > 0 && tid == 0) *mine = s;
            return;
        }
        __syncthreads();
    }

    // Places that stay before this part, and ties that found room in it or earlier.
    int done = s.before, tied = ties_before;
    for (int r = 0; r < rounds; ++r) {
        if (rounds > 1) load(r);
        int mores = 0, same = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            mores += __popcll(__ballot(v[i] > s.found));
            same += __popcll(__ballot(v[i] == s.found));
        }
        if (r) __syncthreads();                                   // (the last round's sums are read)
        if (lane == 0) {
            S.waves[wave] = mores;
            S.ties[wave] = same;
        }
        __syncthreads();
        int all, all_ties;
        int at = done + waves_below(S.waves, wave, lane, &all), met = tied + waves_below(S.ties, wave, lane, &all_ties);
        const int t0 = first_of(r);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool more = v[i] > s.found, tie = v[i] == s.found;
            const uint64_t m = __ballot(more), e = __ballot(tie);
            const int here = met + lower_lanes(e);
            if (more || (tie && here < s.missing)) kept[at + lower_lanes(m) + min(here, s.missing)] = t0 + i * 64;
            at += __popcll(m);
            met += __popcll(e);
        }
        done += all;
        tied += all_ties;
    }
}

// Parts of a sequence and head: as many as fill the chip twice.
static int parts_of(const KVView& c, int B, int64_t max_len) {
    if (max_len <= kWhole) return 1;
    const int64_t want = cdiv(2 * (int64_t)device_cu_count(), (int64_t)B * c.heads);
    return (int)std::max((int64_t)1, std::min({want, cdiv(max_len, kPart), (int64_t)kMostParts}));
}

size_t choose_workspace_bytes(const KVView& c, int B, int64_t max_len) {
    const int parts = parts_of(c, B, max_len);
    if (parts == 1) return 0;
    return align_up((size_t)B * c.heads * parts * (2 * kBins * sizeof(int) + sizeof(ChooseState)), 256);
}

fk_status launch_kv_choose(const KVView& c, const KVChoose& a, int64_t max_len, void* ws, hipStream_t s) {
    const int parts = parts_of(c, a.B, max_len);
    int* counts = (int*)ws;
    const ChooseArgs A{c, a, parts, counts, (ChooseState*)(counts + 2 * (size_t)a.B * c.heads * parts * kBins)};
    const dim3 grid(c.heads, a.B, parts);
    if (parts > 1) {
        kv_choose_kernel<8, 0><<<grid, kChooseThreads, 0, s>>>(A);
        kv_choose_kernel<8, 1><<<grid, kChooseThreads, 0, s>>>(A);
        kv_choose_kernel<8, 2><<<grid, kChooseThreads, 0, s>>>(A);
        kv_choose_kernel<8, 3><<<grid, kChooseThreads, 0, s>>>(A);
    } else if (max_len <= 4 * kChooseThreads) {
        kv_choose_kernel<4, -1><<<grid, kChooseThreads, 0, s>>>(A);
    } else if (max_len <= 8 * kChooseThreads) {
        kv_choose_kernel<8, -1><<<grid, kChooseThreads, 0, s>>>(A);
    } else {                                                      // (longer ones, where there are enough of them, in turns)
        kv_choose_kernel<16, -1><<<grid, kChooseThreads, 0, s>>>(A);
    }
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
