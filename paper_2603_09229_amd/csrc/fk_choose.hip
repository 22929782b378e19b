// Which places of a sequence stay in the 4-bit key/value cache: its first ones, its last ones, and of the others those with the largest weights.
//
// Weights become 32-bit integers of the same order (NaN below all of them).  With m of the middle ones to be kept, the m-th largest value T is
// found 11, 11 and 10 bits at a time, by counting how many of the values that share the bits found so far have which next ones; then
// those above T stay, and of those equal to T the first ones until there are m.  The places are written in ascending order by a prefix
// sum.  Nothing depends on the order in which the counts are added.
//
// A workgroup holds the weights of a sequence and head in registers, read once.  Sequences of more than kWhole tokens are divided among
// workgroups, and the four steps are launches of their own: each counts its part, the next one adds the parts' counts up.
#include <algorithm>

#include "fk_device.h"
#include "fk_evict.h"

namespace fk {

constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr int kWhole = 32 * kChooseThreads;   // most tokens that one workgroup holds in registers
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

// order of weights as integers; 0 is NaN alone
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);                  // (-0 becomes 0)
    return w != w ? 0u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int y = __shfl_up(x, o);
        x += lane >= o ? y : 0;
    }
    return x;
}

// How many of the lanes below this one are in the mask.
__device__ __forceinline__ int lower_lanes(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

struct ChooseShared {
    __align__(16) int bins[kBins][kCopies];
    int waves[kChooseWaves];
    int places[32 * kChooseWaves + 64];  // of a round: places that stay for sure, ties times 2^16, per 64 tokens; then before them
    ChooseState next;
    int ties_before;
    int all;
};

// The bits of the wanted value and what is still wanted below it, from a thread's two counts in descending order; `before_*`: the same counts
// in earlier parts.
__device__ __forceinline__ void find_bin(ChooseShared& S, ChooseState& s, const int (&own)[2], const int (&earlier)[2], int shift, int tid, int* ties_before) {
    const int lane = tid & 63, wave = tid / 64;
    const int sum = own[0] + own[1];
    const int scan = wave_scan(sum, lane);
    if (lane == 63) S.waves[wave] = scan;
    if (tid == 0) {
        S.next = s;
        S.ties_before = 0;
    }
    __syncthreads();
    int above = scan - sum;
#pragma unroll
    for (int w = 0; w < kChooseWaves; ++w) above += w < wave ? S.waves[w] : 0;
    const int hit = above < s.missing && s.missing <= above + own[0] ? 0 : above + own[0] < s.missing && s.missing <= above + sum ? 1 : -1;
    if (hit >= 0) {
        S.next.found = s.found | (uint32_t)(kBins - 1 - 2 * tid - hit) << shift;
        S.next.missing = s.missing - above - (hit ? own[0] : 0);
        S.ties_before = earlier[hit];
    }
    __syncthreads();
    s.found = S.next.found;
    s.missing = S.next.missing;
    *ties_before = S.ties_before;
}

// STAGE -1: everything; 0 to 3: one of four launches over parts.
template <int ITEMS, int STAGE>
__global__ __launch_bounds__(kChooseThreads) void kv_choose_kernel(ChooseArgs A) {
    __shared__ ChooseShared S;
    const KVChoose& a = A.a;
    const KVView& c = A.c;
    const int h = blockIdx.x, b = blockIdx.y, part = STAGE < 0 ? 0 : blockIdx.z, parts = STAGE < 0 ? 1 : A.parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const int len = min(max(a.lens[b], 0), a.max_pages << c.page_shift);
    int32_t* kept = a.kept + ((int64_t)b * c.heads + h) * a.keep;
    if (STAGE <= 0 && h == 0 && part == 0 && tid == 0) a.counts[b] = min(len, a.keep);
    if (len <= a.keep) {
        if (STAGE <= 0)
            for (int64_t j = (int64_t)part * kChooseThreads + tid; j < a.keep; j += (int64_t)parts * kChooseThreads) kept[j] = j < len ? (int)j : -1;
        return;
    }
    const int32_t* table = a.pages + (int64_t)b * a.max_pages;
    const int from = a.first, to = len - a.last;                  // the middle
    const int each = ((len + parts - 1) / parts + kChooseThreads - 1) / kChooseThreads * kChooseThreads;
    const int begin = min((int64_t)part * each, (int64_t)len), end = min((int64_t)begin + each, (int64_t)len);
    const int rounds = (end - begin + ITEMS * kChooseThreads - 1) / (ITEMS * kChooseThreads);

    uint32_t v[ITEMS];
    auto load = [&](int round) {
        int page[ITEMS];
        const int t0 = begin + round * (ITEMS * kChooseThreads) + tid;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) page[i] = table[min(t0 + i * kChooseThreads, len - 1) >> c.page_shift];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int t = min(t0 + i * kChooseThreads, len - 1);
            page[i] = min(max(page[i], 0), (int)c.pages - 1);
            v[i] = order_of(a.mass[(((int64_t)page[i] * c.heads + h) << c.page_shift) + (t & ((1 << c.page_shift) - 1))]);
        }
    };
    auto middle = [&](int t) { return t >= from && t < min(to, end); };
    auto count = [&](const ChooseState& s, int shift, int bits) {
        for (int i = tid; i < kBins * kCopies / 4; i += kChooseThreads) ((uintx4*)S.bins)[i] = uintx4{0, 0, 0, 0};
        __syncthreads();
        for (int r = 0; r < rounds; ++r) {
            if (rounds > 1 || STAGE >= 0 || shift == 21) load(r);
            const int t0 = begin + r * (ITEMS * kChooseThreads) + tid;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (middle(t0 + i * kChooseThreads) && (shift == 21 || (v[i] ^ s.found) >> (shift + bits) == 0))
                    atomicAdd(&S.bins[v[i] >> shift & ((1 << bits) - 1)][lane & (kCopies - 1)], 1);
        }
        __syncthreads();
    };
    // a thread's two counts, of bits 2047 - 2 tid and one less
    auto counted = [&](int (&own)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uintx4 x = *(const uintx4*)S.bins[kBins - 1 - 2 * tid - i];
            own[i] = (int)(x[0] + x[1] + x[2] + x[3]);
        }
    };

    constexpr int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
    ChooseState s{0, a.keep - a.first - a.last, 0};
    int ties_before = 0;
    if constexpr (STAGE < 0) {
        const int none[2] = {0, 0};
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            count(s, shifts[p], widths[p]);
            int own[2];
            counted(own);
            find_bin(S, s, own, none, shifts[p], tid, &ties_before);
        }
    } else {
        const int64_t unit = (int64_t)b * c.heads + h, stage_ints = (int64_t)a.B * c.heads * parts * kBins;
        ChooseState* mine = A.state + unit * parts + part;
        if constexpr (STAGE > 0) {
            if (STAGE > 1) s = *mine;
            const int* all = A.counts + ((STAGE - 1) & 1) * stage_ints + unit * parts * kBins + (kBins - 2 - 2 * tid);
            typedef int intx2 __attribute__((ext_vector_type(2)));
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
            const uint32_t bin = (s.found >> shifts[STAGE - 1]) & ((1u << widths[STAGE - 1]) - 1);
            const uint32_t bin0 = kBins - 1 - 2 * tid;
            int above = (bin0 > bin ? earlier[0] : 0) + (bin0 - 1 > bin && tid < kBins / 2 ? earlier[1] : 0);
            above = wave_scan(above, lane);
            __syncthreads();
            if (lane == 63) S.waves[wave] = above;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kChooseWaves; ++w) s.before += S.waves[w];
            __syncthreads();
        }
        if constexpr (STAGE < 3) {
            count(s, shifts[STAGE], widths[STAGE]);
            int own[2];
            counted(own);
            typedef int intx2 __attribute__((ext_vector_type(2)));
            *(intx2*)(A.counts + (STAGE & 1) * stage_ints + (unit * parts + part) * kBins + (kBins - 2 - 2 * tid)) = intx2{own[1], own[0]};
            if (STAGE > 0 && tid == 0) *mine = s;
            return;
        }
    }

    const bool some = a.keep > a.first + a.last;
    const int ties = s.missing;
    // places that stay before this part: protected ones, larger ones, and the ties that found room
    int done = min(begin, from) + max(begin - max(to, 0), 0) + (some ? s.before : 0), tied = ties_before;
    for (int r = 0; r < rounds; ++r) {
        if (rounds > 1 || STAGE >= 0) load(r);
        const int t0 = begin + r * (ITEMS * kChooseThreads) + tid;
        auto more = [&](int i) {
            const int t = t0 + i * kChooseThreads;
            return (t < end && (t < from || t >= to)) || (some && middle(t) && v[i] > s.found);
        };
        auto tie = [&](int i) { return some && middle(t0 + i * kChooseThreads) && v[i] == s.found; };
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int x = __popcll(__ballot(more(i))) + (__popcll(__ballot(tie(i))) << 16);
            if (lane == 0) S.places[i * kChooseWaves + wave] = x;
        }
        __syncthreads();
        constexpr int ENTRIES = ITEMS * kChooseWaves;             // at most 512, by one wave
        if (wave == 0) {
            constexpr int EACH = (ENTRIES + 63) / 64;
            int x[EACH], sum = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                x[k] = lane * EACH + k < ENTRIES ? S.places[lane * EACH + k] : 0;
                sum += x[k];
            }
            int at = wave_scan(sum, lane);
            if (lane == 63) S.all = at;
            at -= sum;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                S.places[lane * EACH + k] = at;
                at += x[k];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int x = S.places[i * kChooseWaves + wave];
            const bool stays = more(i), equal = tie(i);
            const int met = tied + (int)((uint32_t)x >> 16) + lower_lanes(__ballot(equal));
            if (stays || (equal && met < ties)) kept[done + (x & 0xffff) + lower_lanes(__ballot(stays)) + min(met, ties)] = t0 + i * kChooseThreads;
        }
        const int all = S.all;
        done += all & 0xffff;
        tied += (int)((uint32_t)all >> 16);
        __syncthreads();
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
    } else if (max_len <= 16 * kChooseThreads) {
        kv_choose_kernel<16, -1><<<grid, kChooseThreads, 0, s>>>(A);
    } else {
        kv_choose_kernel<32, -1><<<grid, kChooseThreads, 0, s>>>(A);
    }
    FK_HIP(hipGetLastError());
    return FK_OK;
}

}  // namespace fk
