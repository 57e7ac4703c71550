// The largest logits of every row as (index, value) pairs, and the row's log-sum-exp (ds_top_logits).
//
// One pass over the row: a workgroup keeps a list of candidates in LDS and a bar, a rank that at least k logits seen so far reach; 16 bytes of logits
// below the bar cost one comparison.  When the list grows long, its k best are found, which raises the bar; when a stretch has more logits above the bar
// than the list has room for, the stretch is gone through again, a logit of each thread at a time.  Ranks are unique (the index breaks ties), so neither the
// bar's history nor the order in which threads append shows in the result.  The first bar comes from the first stretch: the m-th best of the largest
// of each wave's 16-byte pieces, m = ceil(k / 4): four times m >= k logits reach the lowest of the four.
//   Few rows are split over workgroups, whose lists and sums go through work_dev to a second launch.
// Bound by reading the logits once where there are many rows.
#include "dsq_answers.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kRoom = 1024, kLong = 512;                     // candidates the list has room for, and from which on it is shortened
constexpr int kPieces = 4;                                        // 16-byte pieces of a thread in a stretch
constexpr uint64_t kRowsOfLaunch = 1u << 22;                      // a launch dimension holds fewer than 2^32 work-items

struct TopShape : LogitsArgs {
    uint32_t parts;                                               // workgroups of a row
    uint64_t part_logits;                                         // a multiple of a stretch
    uint64_t row0;
    uint64_t* lists;                                              // [row][part][kLong] ranks
    struct Part {
        float max, sum;
        uint32_t held, unused;                                    // ranks in the list
    };
    Part* found;                                                  // [row][part]
};

struct TopLds {
    uint64_t list[kRoom];
    uint32_t bins[256];
    uint64_t edges[2][kWaves];
    uint32_t totals[kWaves];
    float sums[2 * kWaves];
    uint32_t count;                                               // of the list
    uint32_t bin, above, inside;                                  // kth_rank: the k-th's bin, ranks in higher ones and in it
};

__device__ __forceinline__ uint64_t wave_max_rank(uint64_t v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t other = __shfl_xor((unsigned long long)v, o);
        v = other > v ? other : v;
    }
    return v;
}

// A number that exactly k of the list's n > k ranks reach.  Eight bits at a time from the first in which ranks differ: a histogram of those that agree with
// what is known of the k-th, and the bin in which the k-th lies.
__device__ uint64_t kth_rank(TopLds& s, uint32_t n, uint32_t k) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint64_t mine[kRoom / kThreads], high = 0, low = ~0ull;
#pragma unroll
    for (uint32_t q = 0; q < kRoom / kThreads; ++q) {
        const uint32_t at = q * kThreads + threadIdx.x;
        mine[q] = at < n ? s.list[at] : 0;                        // (0 is no rank)
        high = mine[q] > high ? mine[q] : high;
        if (at < n) low = mine[q] < low ? mine[q] : low;
    }
    high = wave_max_rank(high);
    low = ~wave_max_rank(~low);
    if (lane == 0) {
        s.edges[0][wave] = high;
        s.edges[1][wave] = low;
    }
    s.bins[threadIdx.x] = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        high = s.edges[0][w] > high ? s.edges[0][w] : high;
        low = s.edges[1][w] < low ? s.edges[1][w] : low;
    }
    int shift = 64 - __builtin_clzll(high ^ low);                 // the bits from here on are the same in all (n > 1: some differ)
    uint64_t known = shift == 64 ? 0 : high >> shift << shift;
    for (;;) {
        const int next = shift > 8 ? shift - 8 : 0;
#pragma unroll
        for (uint32_t q = 0; q < kRoom / kThreads; ++q)
            if (mine[q] && (shift == 64 || mine[q] >> shift == known >> shift)) atomicAdd(&s.bins[mine[q] >> next & ((1u << (shift - next)) - 1)], 1u);
        __syncthreads();
        // thread i has bin 255 - i: what lies in it and above
        const uint32_t bin = 255 - threadIdx.x, here = s.bins[bin];
        uint32_t upto = here;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t other = (uint32_t)__shfl_up((int)upto, o);
            if (lane >= (uint32_t)o) upto += other;
        }
        if (lane == 63) s.totals[wave] = upto;
        __syncthreads();
        s.bins[bin] = 0;
        for (uint32_t w = 0; w < wave; ++w) upto += s.totals[w];
        if (upto >= k && upto - here < k) {
            s.bin = bin;
            s.above = upto - here;
            s.inside = here;
        }
        __syncthreads();
        known |= (uint64_t)s.bin << next;
        k -= s.above;
        const bool all = s.inside == k;                           // all of the bin: nothing below matters
        shift = next;
        if (all || shift == 0) return known;
        __syncthreads();                                          // (s.bin is written again)
    }
}

// Leaves the k best of the list's n > k ranks in its first places, in no order; returns the lowest of them.
__device__ uint64_t keep_best(TopLds& s, uint32_t n, uint32_t k) {
    const uint64_t bar = kth_rank(s, n, k);
    uint64_t mine[kRoom / kThreads];
#pragma unroll
    for (uint32_t q = 0; q < kRoom / kThreads; ++q) mine[q] = q * kThreads + threadIdx.x < n ? s.list[q * kThreads + threadIdx.x] : 0;
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t q = 0; q < kRoom / kThreads; ++q)
        if (mine[q] >= bar) s.list[atomicAdd(&s.count, 1u)] = mine[q];
    __syncthreads();
    return bar;
}

// The list's best k (all of it where it holds fewer) as pairs in ascending index order.
template <typename F>
__device__ void write_pairs(TopLds& s, uint32_t n, uint32_t k, F value) {
    if (n > k) (void)keep_best(s, n, k);
    for (uint32_t q = threadIdx.x; q < k; q += kThreads) {
        const uint64_t rank = s.list[q];
        const uint32_t mine = (uint32_t)rank;                     // the index's complement
        uint32_t place = 0;
        for (uint32_t i = 0; i < k; ++i) place += (uint32_t)s.list[i] > mine ? 1u : 0u;
        value(place, ~mine);
    }
}

// A wave's lower bound for its m-th largest key: the largest number that m of its lanes' keys (kPieces each) reach.
__device__ uint32_t wave_bar(const uint32_t (&key)[kPieces], uint32_t m) {
    uint32_t bar = 0;
    for (uint32_t bit = 0x80000000u; bit > 0x8000u; bit >>= 1) {  // sixteen bits of it will do
        uint32_t c = 0;
#pragma unroll
        for (int q = 0; q < kPieces; ++q) c += (uint32_t)__popcll(__ballot(key[q] >= (bar | bit)));
        if (c >= m) bar |= bit;
    }
    return bar;
}

__device__ __forceinline__ float row_lse(Spread s, float scale, float temperature) {
    const LogSum l = log_sum(s, scale);
    return l.from / temperature + l.rest;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) top_logits_kernel(TopShape a) {
    constexpr uint32_t E = Pieces<T>::E, kStretch = kThreads * kPieces * E;
    using Piece = typename Pieces<T>::Piece;
    __shared__ TopLds s;
    const uint64_t row = a.row0 + blockIdx.x;
    const uint32_t k = a.k, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    const uint64_t begin = (uint64_t)blockIdx.y * a.part_logits, end = begin + a.part_logits < a.vocab ? begin + a.part_logits : a.vocab;
    const float scale = kLog2e / a.temperature;
    Spread spread = kNoSpread;
    uint64_t bar = 0;                                             // candidates: ranks above it
    float bar_value = -__builtin_huge_valf();                     // logits below it are no candidates
    bool first = true;
    if (threadIdx.x == 0) s.count = 0;
    uint32_t held = 0;                                            // in the list; the same in every thread
    __syncthreads();

    for (uint64_t at = begin; at < end; at += kStretch) {
        // element e of piece p: column at + (p kThreads + thread) E + e; -inf behind the end, which is never asked for
        float v[kPieces][E];
        const uint64_t mine = at + (uint64_t)threadIdx.x * E;
        if (at + kStretch <= end) {
            Piece raw[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) raw[p] = *reinterpret_cast<const Piece*>(z + mine + (uint64_t)p * kThreads * E);
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) v[p][e] = (float)raw[p][e];
        } else {
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) {
                    const uint64_t c = mine + (uint64_t)p * kThreads * E + e;
                    v[p][e] = c < end ? (float)z[c] : -__builtin_huge_valf();
                }
        }
        auto there = [&](int p, uint32_t e) { return mine + (uint64_t)p * kThreads * E + e < end; };
        auto rank_of = [&](int p, uint32_t e) { return logit_rank(v[p][e], (uint32_t)(mine + (uint64_t)p * kThreads * E + e)); };
        float most[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) most[p] = largest_of(v[p]);
        add_logits(spread, v, largest_of(most), scale);
        if (first && end - at >= (uint64_t)kThreads * kPieces * E) {
            uint32_t key[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) key[p] = logit_key(most[p]);
            const uint32_t b = wave_bar(key, (k + kWaves - 1) / kWaves);
            if (lane == 0) s.totals[wave] = b;
            __syncthreads();
            uint32_t lowest = s.totals[0];
            for (int w = 1; w < kWaves; ++w) lowest = s.totals[w] < lowest ? s.totals[w] : lowest;
            __syncthreads();
            if (lowest > 0) bar = ((uint64_t)(lowest - 1) << 32) | 0xFFFFFFFFull;         // everything of that key or a higher one passes
        }
        first = false;
        auto bar_to_value = [&] {
            const uint32_t key = (uint32_t)(bar >> 32);
            const uint32_t bits = key & 0x80000000u ? key & 0x7FFFFFFFu : ~key;
            bar_value = bar == 0 ? -__builtin_huge_valf() : __uint_as_float(bits);
        };
        bar_to_value();
        // a logit passes if it is not below the bar's value (NaN passes) and its rank is above the bar
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
            if (!(most[p] < bar_value))
#pragma unroll
                for (uint32_t e = 0; e < E; ++e)
                    if (!(v[p][e] < bar_value)) {
                        const uint64_t rank = rank_of(p, e);
                        if (rank > bar && there(p, e)) {
                            const uint32_t place = atomicAdd(&s.count, 1u);
                            if (place < kRoom) s.list[place] = rank;
                        }
                    }
        __syncthreads();
        const uint32_t count = s.count;
        __syncthreads();
        if (count <= kRoom) {
            held = count;
            if (held > kLong) {                                   // (k <= 256: twice as many at least)
                bar = keep_best(s, held, k);
                held = k;
            }
            continue;
        }
        // too many: back to what was held, and one element of each thread at a time
        if (threadIdx.x == 0) s.count = held;
        __syncthreads();
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) {
                if (held + kThreads > kRoom) {
                    bar = keep_best(s, held, k);
                    held = k;
                }
                const uint64_t rank = rank_of(p, e);
                if (rank > bar && there(p, e)) s.list[atomicAdd(&s.count, 1u)] = rank;
                __syncthreads();
                held = s.count;
                __syncthreads();
            }
    }
    spread = workgroup_spread<kWaves>(spread, scale, s.sums);
    __syncthreads();
    if (a.parts == 1) {
        write_pairs(s, held, k, [&](uint32_t place, uint32_t index) { a.pairs[row * k + place] = make_uint2(index, __float_as_uint((float)z[index])); });
        if (a.lse && threadIdx.x == 0) a.lse[row] = row_lse(spread, scale, a.temperature);
        return;
    }
    if (held > kLong) {
        (void)keep_best(s, held, k);
        held = k;
    }
    const uint64_t part = row * a.parts + blockIdx.y;
    for (uint32_t q = threadIdx.x; q < held; q += kThreads) a.lists[part * kLong + q] = s.list[q];
    if (threadIdx.x == 0) a.found[part] = {spread.max, spread.sum, held, 0};
}

// Joins the parts of a row.
template <typename T>
__global__ void __launch_bounds__(kThreads) top_logits_join_kernel(TopShape a) {
    __shared__ TopLds s;
    const uint64_t row = a.row0 + blockIdx.x;
    const uint32_t k = a.k;
    const TopShape::Part* found = a.found + row * a.parts;
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    uint32_t held = 0;
    uint64_t bar = 0;
    for (uint32_t p = 0; p < a.parts; ++p) {
        const uint64_t* list = a.lists + (row * a.parts + p) * kLong;
        const uint32_t n = found[p].held;
        if (held + n > kRoom) {                                   // (n <= 512, k <= 256)
            bar = keep_best(s, held, k);
            held = k;
        }
        for (uint32_t q = threadIdx.x; q < n; q += kThreads)
            if (list[q] > bar) s.list[atomicAdd(&s.count, 1u)] = list[q];
        __syncthreads();
        held = s.count;
        __syncthreads();
    }
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    write_pairs(s, held, k, [&](uint32_t place, uint32_t index) { a.pairs[row * k + place] = make_uint2(index, __float_as_uint((float)z[index])); });
    if (!a.lse) return;
    const float scale = kLog2e / a.temperature;
    Spread spread = kNoSpread;
    for (uint32_t p = threadIdx.x; p < a.parts; p += kThreads) {
        const TopShape::Part v = found[p];
        spread = join(spread, Spread{v.max, v.sum}, scale);
    }
    spread = workgroup_spread<kWaves>(spread, scale, s.sums);
    if (threadIdx.x == 0) a.lse[row] = row_lse(spread, scale, a.temperature);
}

// Workgroups of a row: as many as fill the GPU, each with a stretch or more.
template <typename T>
void top_plan(uint64_t rows, uint64_t vocab, uint32_t& parts, uint64_t& part_logits) {
    constexpr uint64_t stretch = kThreads * kPieces * (16 / sizeof(T));
    const uint64_t stretches = (vocab + stretch - 1) / stretch;
    uint64_t p = rows >= 512 ? 1 : 1024 / rows;
    if (p > stretches) p = stretches;
    if (p > 64) p = 64;
    if (p < 1) p = 1;
    const uint64_t each = (stretches + p - 1) / p;
    part_logits = each * stretch;
    parts = (uint32_t)((stretches + each - 1) / each);
}


template <typename T>
void launch_top_of(const LogitsArgs& args, hipStream_t stream) {
    TopShape a{};
    static_cast<LogitsArgs&>(a) = args;
    top_plan<T>(a.rows, a.vocab, a.parts, a.part_logits);
    a.lists = static_cast<uint64_t*>(a.work);
    a.found = reinterpret_cast<TopShape::Part*>(a.lists + a.rows * a.parts * kLong);
    for (uint64_t r = 0; r < a.rows; r += kRowsOfLaunch) {
        a.row0 = r;
        const unsigned here = (unsigned)(a.rows - r < kRowsOfLaunch ? a.rows - r : kRowsOfLaunch);
        hipLaunchKernelGGL(top_logits_kernel<T>, dim3(here, a.parts), dim3(kThreads), 0, stream, a);
        if (a.parts > 1) hipLaunchKernelGGL(top_logits_join_kernel<T>, dim3(here), dim3(kThreads), 0, stream, a);
    }
}

}  // namespace

uint64_t top_logits_work_bytes(const ds_logits& l) {
    uint32_t parts = 1;
    uint64_t part_logits;
    by_dtype(l.dtype, [&](auto kind) { top_plan<decltype(kind)>(l.rows, l.vocab, parts, part_logits); });
    return parts > 1 ? l.rows * parts * (kLong * sizeof(uint64_t) + sizeof(TopShape::Part)) : 0;
}

hipError_t launch_top_logits(const LogitsArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_top_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
