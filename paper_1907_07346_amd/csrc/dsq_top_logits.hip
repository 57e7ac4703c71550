// The largest logits of every row as (index, value) pairs, and the row's log-sum-exp (ds_top_logits).
//
// One pass over the row: a workgroup keeps a list of candidates in LDS and a bar, a rank that at least k logits seen so far reach; a logit
// below the bar costs one comparison.  When a stretch has more logits above the bar than the list has room for, the k best of the list are
// found, which raises the bar, and the stretch is gone through again, a few logits of each thread at a time.  Ranks are unique (the index breaks ties), so neither the bar's
// history nor the order in which threads append shows in the result.  The first bar comes from the first stretch: each wave's m-th best of its 16-byte pieces' maxima, m = ceil(k / 4):
// four times m >= k logits reach the lowest of the four.
// Few rows are split over workgroups, whose lists of k and sums go through work_dev to a second launch.
// Bound by reading the logits once where there are many rows.
#include "dsq_answers.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kRoom = 1024;                                  // candidates in the list
constexpr int kPieces = 4;                                        // 16-byte pieces of a thread in a stretch
constexpr uint64_t kRowsOfLaunch = 1u << 22;                      // a launch dimension holds fewer than 2^32 work-items

struct TopShape : LogitsArgs {
    uint32_t parts;                                               // workgroups of a row
    uint64_t part_logits;                                         // a multiple of a stretch
    uint64_t row0;
    uint64_t* lists;                                              // [row][part][k] ranks, 0 where a part has fewer
    float2* spreads;                                              // [row][part]
};

struct TopLds {
    uint64_t list[kRoom];
    uint32_t counts[2][kWaves];
    uint64_t edges[2][kWaves];
    float sums[2 * kWaves];
    uint32_t count;
};

__device__ __forceinline__ uint64_t wave_max_rank(uint64_t v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t other = __shfl_xor((unsigned long long)v, o);
        v = other > v ? other : v;
    }
    return v;
}

// The rank that exactly k of the list's n > k ranks reach: halving between the lowest and the highest, by counts.
__device__ uint64_t kth_rank(TopLds& s, uint32_t n, uint32_t k) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint64_t mine[kRoom / kThreads], high = 0, low = ~0ull;
#pragma unroll
    for (uint32_t q = 0; q < kRoom / kThreads; ++q) {
        const uint32_t at = q * kThreads + threadIdx.x;
        mine[q] = at < n ? s.list[at] : 0;
        high = mine[q] > high ? mine[q] : high;
        if (at < n) low = mine[q] < low ? mine[q] : low;
    }
    high = wave_max_rank(high);
    low = ~wave_max_rank(~low);
    if (lane == 0) {
        s.edges[0][wave] = high;
        s.edges[1][wave] = low;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        high = s.edges[0][w] > high ? s.edges[0][w] : high;
        low = s.edges[1][w] < low ? s.edges[1][w] : low;
    }
    // more than k reach low, and, where k > 1, fewer than k reach high
    uint64_t found = high;
    for (uint32_t turn = 0; high - low > 1; ++turn) {
        const uint64_t mid = low + (high - low) / 2;
        uint32_t c = 0;
#pragma unroll
        for (uint32_t q = 0; q < kRoom / kThreads; ++q) c += (uint32_t)__popcll(__ballot(mine[q] >= mid));
        if (lane == 0) s.counts[turn & 1][wave] = c;
        __syncthreads();
        c = 0;
        for (int w = 0; w < kWaves; ++w) c += s.counts[turn & 1][w];
        found = mid;
        if (c == k) break;
        if (c > k) low = mid;
        else high = mid;
        found = high;
    }
    return found;
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
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
        uint32_t c = 0;
#pragma unroll
        for (int q = 0; q < kPieces; ++q) c += (uint32_t)__popcll(__ballot(key[q] >= (bar | bit)));
        if (c >= m) bar |= bit;
    }
    return bar;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) top_logits_kernel(TopShape a) {
    constexpr uint32_t E = 16 / sizeof(T), kStretch = kThreads * kPieces * E;
    typedef T Piece __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    __shared__ TopLds s;
    const uint64_t row = a.row0 + blockIdx.x;
    const uint32_t k = a.k, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    const uint64_t begin = (uint64_t)blockIdx.y * a.part_logits, end = begin + a.part_logits < a.vocab ? begin + a.part_logits : a.vocab;
    const float scale = kLog2e / a.temperature;
    const bool sums = a.lse != nullptr;
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
        for (int p = 0; p < kPieces; ++p) {
            most[p] = v[p][0];
#pragma unroll
            for (uint32_t e = 1; e < E; ++e) most[p] = fmaxf(most[p], v[p][e]);
        }
        if (sums) {
            float m = spread.max;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) m = fmaxf(m, most[p]);
            const float r = reference(m);
            float total = 0.f;
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) total += power2((v[p][e] - r) * scale);
            if (spread.sum != 0.f) total = fmaf(spread.sum, exp2f((reference(spread.max) - r) * scale), total);
            spread = {m, total};
        }
        if (first && end - at >= (uint64_t)kThreads * kPieces * E) {
            uint32_t key[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) key[p] = logit_key(most[p]);                 // (NaN beside a number: the number's, which is lower)
            const uint32_t b = wave_bar(key, (k + kWaves - 1) / kWaves);
            if (lane == 0) s.counts[0][wave] = b;
            __syncthreads();
            uint32_t lowest = s.counts[0][0];
            for (int w = 1; w < kWaves; ++w) lowest = s.counts[0][w] < lowest ? s.counts[0][w] : lowest;
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
        uint32_t passed = 0;
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (!(v[p][e] < bar_value)) passed |= 1u << (p * E + e);
        if (passed) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e)
                    if (passed >> (p * E + e) & 1) {
                        const uint64_t rank = rank_of(p, e);
                        if (rank > bar && there(p, e)) {
                            const uint32_t place = atomicAdd(&s.count, 1u);
                            if (place < kRoom) s.list[place] = rank;
                        }
                    }
        }
        __syncthreads();
        const uint32_t count = s.count;
        __syncthreads();
        if (count <= kRoom) {
            held = count;
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
    if (sums) spread = workgroup_spread<kWaves>(spread, scale, s.sums);
    __syncthreads();
    if (a.parts == 1) {
        write_pairs(s, held, k, [&](uint32_t place, uint32_t index) { a.pairs[row * k + place] = make_uint2(index, __float_as_uint((float)z[index])); });
        if (sums && threadIdx.x == 0) a.lse[row] = spread_lse(spread, a.temperature);
        return;
    }
    if (held > k) {
        (void)keep_best(s, held, k);
        held = k;
    }
    const uint64_t list = row * a.parts + blockIdx.y;
    for (uint32_t q = threadIdx.x; q < k; q += kThreads) a.lists[list * k + q] = q < held ? s.list[q] : 0;
    if (threadIdx.x == 0) a.spreads[list] = make_float2(spread.max, spread.sum);
}

// Joins the parts of a row.
template <typename T>
__global__ void __launch_bounds__(kThreads) top_logits_join_kernel(TopShape a) {
    __shared__ TopLds s;
    const uint64_t row = a.row0 + blockIdx.x;
    const uint32_t k = a.k;
    const uint64_t* lists = a.lists + row * a.parts * k;
    const uint32_t all = a.parts * k;
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    uint32_t held = 0;
    uint64_t bar = 0;
    for (uint32_t at = 0; at < all; at += kThreads) {
        if (held + kThreads > kRoom) {
            bar = keep_best(s, held, k);
            held = k;
        }
        const uint64_t rank = at + threadIdx.x < all ? lists[at + threadIdx.x] : 0;
        if (rank > bar) s.list[atomicAdd(&s.count, 1u)] = rank;
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
        const float2 v = a.spreads[row * a.parts + p];
        spread = join(spread, Spread{v.x, v.y}, scale);
    }
    spread = workgroup_spread<kWaves>(spread, scale, s.sums);
    if (threadIdx.x == 0) a.lse[row] = spread_lse(spread, a.temperature);
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

uint64_t spreads_at(uint64_t lists) { return lists * sizeof(uint64_t); }

template <typename T>
void launch_top_of(const LogitsArgs& args, hipStream_t stream) {
    TopShape a{};
    static_cast<LogitsArgs&>(a) = args;
    top_plan<T>(a.rows, a.vocab, a.parts, a.part_logits);
    a.lists = static_cast<uint64_t*>(a.work);
    a.spreads = reinterpret_cast<float2*>(static_cast<uint8_t*>(a.work) + spreads_at(a.rows * a.parts * a.k));
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
    return parts > 1 ? spreads_at(l.rows * parts * l.k) + l.rows * parts * sizeof(float2) : 0;
}

hipError_t launch_top_logits(const LogitsArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_top_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
