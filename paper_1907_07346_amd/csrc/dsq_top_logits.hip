// The largest logits of every row as (index, value) pairs, and the row's log-sum-exp (ds_top_logits).
//
// One pass over the row: a workgroup keeps a list of candidates in LDS and a bar, a rank that at least k logits seen so far reach; 16 bytes of logits
// below the bar cost one comparison.  When the list grows long, its k best are found, which raises the bar; when a stretch has more logits above the bar
// than the list has room for, the stretch is gone through again, a logit of each thread at a time.  Ranks are unique (the index breaks ties), so neither the
// bar's history nor the order in which threads append shows in the result.  The first bar comes from the first stretch: the m-th best of the largest
// of each wave's 16-byte pieces, m = ceil(k / 4): four times m >= k logits reach the lowest of the four, or it is minus infinity, which stands for what
// is behind the end, and all pass.
//   Few rows are split over workgroups, whose lists and sums go through work_dev to a second launch, which has room for all of a row's lists at once
// (1 x 1000000, k = 100, fp32: 33.8 us; 72 where lists came one after the other).  Those two launches are mostly waiting: 1 x 131072, k = 64, bf16, 6.0 + 8.6 us,
// where an empty launch takes 2; what the first finds is some 1500 candidates, and the second's time is three reads of memory, one behind the other, one
// histogram and the ranks in one of its bins.
//   Many rows: 2048 x 65536, fp32, k = 128, 111 us alone and 105 a call among others, 5.1 TB/s, with the vector units busy 65 % of the time; a row is a workgroup's,
// and 1000 rows take 58.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kRoom = 1024, kLong = 512;                     // candidates the list has room for, and from which on it is shortened
constexpr uint32_t kJoinRoom = 4096;                              // candidates of a row's parts
constexpr int kPieces = 4;                                        // 16-byte pieces of a thread in a stretch
constexpr uint64_t kRowsOfLaunch = 1u << 22;                      // a launch dimension holds fewer than 2^32 work-items

struct TopShape : LogitsArgs {
    uint32_t parts;                                               // workgroups of a row
    uint64_t part_logits;                                         // a multiple of a stretch
    uint64_t row0;
    uint32_t room;                                                // of a part's list, at least k
    uint64_t* lists;                                              // [row][part][room] ranks
    struct Part {
        float max, sum;
        uint32_t held, unused;                                    // ranks in the list
    };
    Part* found;                                                  // [row][part]
};

template <uint32_t ROOM>
struct TopLds {
    uint64_t list[ROOM];
    uint32_t bins[256];
    uint64_t edges[2][kWaves];
    uint32_t totals[kWaves];
    float sums[2 * kWaves];
    uint32_t count;                                               // of the list
    uint32_t bin, above, inside, gathered;                        // kth_rank: the k-th's bin, ranks in higher ones and in it ...
    uint64_t few[kThreads], kth;                                  // ... and those in it, where they are few
};

// The k-th largest of n <= kThreads ranks: a thread for each counts those above its own.
template <uint32_t ROOM>
__device__ __forceinline__ uint64_t kth_of_few(TopLds<ROOM>& s, const uint64_t* few, uint32_t n, uint32_t k) {
    const uint64_t rank = threadIdx.x < n ? few[threadIdx.x] : 0;
    uint32_t higher = 0;
#pragma unroll 8
    for (uint32_t i = 0; i < n; ++i) higher += few[i] > rank ? 1u : 0u;
    if (threadIdx.x < n && higher == k - 1) s.kth = rank;
    __syncthreads();
    return s.kth;
}

// A number that exactly k of the list's n > k ranks reach.  Up to eight bits at a time, of those in which ranks differ: a histogram of the ranks that agree
// with what is known of the k-th, and the bin in which the k-th lies, until there is a thread for each rank in the bin.
template <uint32_t ROOM>
__device__ uint64_t kth_rank(TopLds<ROOM>& s, uint32_t n, uint32_t k) {
    if (n <= kThreads) return kth_of_few(s, s.list, n, k);        // (8 x 32003, k = 16, fp16: 17.8 us without it, 15.4 with it)
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint64_t mine[ROOM / kThreads], some = 0, all = ~0ull;
#pragma unroll
    for (uint32_t q = 0; q < ROOM / kThreads; ++q) {
        const uint32_t at = q * kThreads + threadIdx.x;
        mine[q] = at < n ? s.list[at] : 0;                        // (0 is no rank)
        some |= mine[q];
        all &= at < n ? mine[q] : ~0ull;
    }
    auto either = [](uint32_t a, uint32_t b) { return a | b; };
    auto both = [](uint32_t a, uint32_t b) { return a & b; };
    some = (uint64_t)over_lanes<64>((uint32_t)(some >> 32), either) << 32 | over_lanes<64>((uint32_t)some, either);
    all = (uint64_t)over_lanes<64>((uint32_t)(all >> 32), both) << 32 | over_lanes<64>((uint32_t)all, both);
    if (lane == 0) {
        s.edges[0][wave] = some;
        s.edges[1][wave] = all;
    }
    s.bins[threadIdx.x] = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        some |= s.edges[0][w];
        all &= s.edges[1][w];
    }
    uint64_t open = some ^ all, known = all;                      // bits in which ranks differ and that are not known yet (n > 1: some); the k-th's others
    for (;;) {
        const int top = 64 - __builtin_clzll(open), next = top > 8 ? top - 8 : 0;
        const uint64_t fixed = top == 64 ? 0 : ~0ull << top;
#pragma unroll
        for (uint32_t q = 0; q < ROOM / kThreads; ++q)
            if (mine[q] && ((mine[q] ^ known) & fixed) == 0) atomicAdd(&s.bins[mine[q] >> next & 255u & ((1u << (top - next)) - 1)], 1u);
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
        const uint64_t digit = ((1ull << (top - next)) - 1) << next;
        known = (known & ~digit) | (uint64_t)s.bin << next;
        open &= ~digit & ~fixed;
        k -= s.above;
        const bool whole = s.inside == k;                         // all of the bin: nothing below matters, and known has no open bit set
        if (whole || open == 0) return known;
        const uint32_t inside = s.inside;
        if (threadIdx.x == 0) s.gathered = 0;
        __syncthreads();                                          // (s.bin is written again)
        if (inside > kThreads) continue;
        const uint64_t same = ~0ull << next;
#pragma unroll
        for (uint32_t q = 0; q < ROOM / kThreads; ++q)
            if (mine[q] && ((mine[q] ^ known) & same) == 0) s.few[atomicAdd(&s.gathered, 1u)] = mine[q];
        __syncthreads();
        return kth_of_few(s, s.few, inside, k);
    }
}

// Leaves the k best of the list's n > k ranks in its first places, in no order; returns the lowest of them.
template <uint32_t ROOM>
__device__ uint64_t keep_best(TopLds<ROOM>& s, uint32_t n, uint32_t k) {
    const uint64_t bar = kth_rank(s, n, k);
    uint64_t mine[ROOM / kThreads];
#pragma unroll
    for (uint32_t q = 0; q < ROOM / kThreads; ++q) mine[q] = q * kThreads + threadIdx.x < n ? s.list[q * kThreads + threadIdx.x] : 0;
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t q = 0; q < ROOM / kThreads; ++q)
        if (mine[q] >= bar) s.list[atomicAdd(&s.count, 1u)] = mine[q];
    __syncthreads();
    return bar;
}

// The list's best k (all of it where it holds fewer) as pairs in ascending index order.  A rank tells its logit, but not which zero or NaN it is.
template <typename T, uint32_t ROOM>
__device__ void write_pairs(TopLds<ROOM>& s, uint32_t n, uint32_t k, const T* z, uint2* pairs) {
    if (n > k) (void)keep_best(s, n, k);
    for (uint32_t q = threadIdx.x; q < k; q += kThreads) {
        const uint64_t rank = s.list[q];
        const uint32_t mine = (uint32_t)rank, key = (uint32_t)(rank >> 32);                // (mine: the index's complement)
        uint32_t bits = key & 0x80000000u ? key & 0x7FFFFFFFu : ~key, place = 0;
        if (bits == 0 || key == logit_key(__builtin_nanf(""))) bits = __float_as_uint((float)z[~mine]);
#pragma unroll 8
        for (uint32_t i = 0; i < k; ++i) place += (uint32_t)s.list[i] > mine ? 1u : 0u;
        pairs[place] = make_uint2(~mine, bits);
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
    __shared__ TopLds<kRoom> s;
    __shared__ u32x4 pieces[kPieces][kThreads];                   // of the thread: those with candidates
    const uint64_t row = a.row0 + blockIdx.x;
    const uint32_t k = a.k, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    const uint64_t begin = (uint64_t)blockIdx.y * a.part_logits, end = begin + a.part_logits < a.vocab ? begin + a.part_logits : a.vocab;
    const float scale = kLog2e / a.temperature;
    Spread spread = kNoSpread;
    uint64_t bar = 0;                                             // candidates: ranks above it
    float bar_value = -kInf;                                      // logits below it are no candidates
    auto raise = [&](uint64_t to) {
        bar = to;
        const uint32_t key = (uint32_t)(bar >> 32), bits = key & 0x80000000u ? key & 0x7FFFFFFFu : ~key;
        bar_value = __uint_as_float(bits);
    };
    if (threadIdx.x == 0) s.count = 0;
    uint32_t held = 0;                                            // in the list; the same in every thread
    __syncthreads();

    // Element e of piece p of a stretch: column at + (p kThreads + thread) E + e; what lies behind the end counts as minus infinity, and is no candidate.
    auto fetch = [&](Piece (&raw)[kPieces], uint64_t at) {
        const T* from = z + at + (uint64_t)threadIdx.x * E;
        if (at + kStretch <= end) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) raw[p] = *reinterpret_cast<const Piece*>(from + (uint64_t)p * kThreads * E);
        } else {
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) {
                    const uint64_t c = at + ((uint64_t)p * kThreads + threadIdx.x) * E + e;
                    raw[p][e] = c < end ? z[c] : (T)-kInf;
                }
        }
    };
    auto go_through = [&](const Piece (&raw)[kPieces], uint64_t at, bool set_bar) {
        float v[kPieces][E], most[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) v[p][e] = (float)raw[p][e];
            most[p] = largest_of(v[p]);
        }
        add_logits(spread, v, largest_of(most), scale);
        if (set_bar) {
            uint32_t key[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) key[p] = logit_key(most[p]);
            const uint32_t b = wave_bar(key, (k + kWaves - 1) / kWaves);
            if (lane == 0) s.totals[wave] = b;
            __syncthreads();
            uint32_t lowest = s.totals[0];
            for (int w = 1; w < kWaves; ++w) lowest = s.totals[w] < lowest ? s.totals[w] : lowest;
            __syncthreads();
            if (lowest > 0) raise(((uint64_t)(lowest - 1) << 32) | 0xFFFFFFFFull);        // everything of that key or a higher one passes
        }
        // a logit passes if it is not below the bar's value (NaN passes) and its rank is above the bar
        uint32_t passed = 0;
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
            if (!(most[p] < bar_value))
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) passed |= v[p][e] < bar_value ? 0u : 1u << (p * E + e);
        // few: their pieces go into LDS, where a logit has an address (read from memory once more: 2048 x 65536, fp32, k = 128, 13 us more)
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
            if (!(most[p] < bar_value)) pieces[p][threadIdx.x] = __builtin_bit_cast(u32x4, raw[p]);
        while (passed) {
            const uint32_t bit = __builtin_ctz(passed);
            passed &= passed - 1;
            const uint64_t column = at + ((uint64_t)(bit / E) * kThreads + threadIdx.x) * E + bit % E;
            if (column >= end) continue;
            const uint64_t rank = logit_rank((float)reinterpret_cast<const T*>(&pieces[bit / E][threadIdx.x])[bit % E], (uint32_t)column);
            if (rank <= bar) continue;
            const uint32_t place = atomicAdd(&s.count, 1u);
            if (place < kRoom) s.list[place] = rank;
        }
    };
    // fp32 has registers for the next stretch's logits on their way meanwhile: 1000 x 65536, k = 128, 57.6 us, 59.8 without; dtypes of 16 bits, whose stretches
    // are twice as many numbers, have not: 300 x 50000, k = 100, fp16, 20.3 without, 23.5 with them.
    constexpr bool kAhead = sizeof(T) == 4;
    Piece coming[kPieces];
    if (kAhead) fetch(coming, begin);
    for (uint64_t at = begin; at < end; at += kStretch) {
        Piece raw[kPieces];
        if constexpr (kAhead) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) raw[p] = coming[p];
            if (at + kStretch < end) fetch(coming, at + kStretch);
            __builtin_amdgcn_sched_barrier(0);
        } else {
            fetch(raw, at);
        }
        go_through(raw, at, at == begin);
        __syncthreads();
        const uint32_t count = s.count;
        __syncthreads();
        if (count <= kRoom) {
            held = count;
            if (held > kLong) {                                   // (k <= 256: twice as many at least)
                raise(keep_best(s, held, k));
                held = k;
            }
            continue;
        }
        // too many: back to what was held, and a logit of each thread at a time
        if (threadIdx.x == 0) s.count = held;
        __syncthreads();
        const uint64_t to = at + kStretch < end ? at + kStretch : end;
        for (uint64_t from = at; from < to; from += kThreads) {
            if (held + kThreads > kRoom) {
                raise(keep_best(s, held, k));
                held = k;
            }
            const uint64_t column = from + threadIdx.x;
            if (column < to) {
                const uint64_t rank = logit_rank((float)z[column], (uint32_t)column);
                if (rank > bar) s.list[atomicAdd(&s.count, 1u)] = rank;
            }
            __syncthreads();
            held = s.count;
            __syncthreads();
        }
    }
    spread = workgroup_spread<kWaves>(spread, scale, s.sums);
    __syncthreads();
    if (a.parts == 1) {
        write_pairs(s, held, k, z, a.pairs + row * k);
        if (a.lse && threadIdx.x == 0) a.lse[row] = row_lse(spread, scale, a.temperature);
        return;
    }
    if (held > a.room) {
        (void)keep_best(s, held, k);
        held = k;
    }
    const uint64_t part = row * a.parts + blockIdx.y;
    for (uint32_t q = threadIdx.x; q < held; q += kThreads) a.lists[part * a.room + q] = s.list[q];
    if (threadIdx.x == 0) a.found[part] = {spread.max, spread.sum, held, 0};
}

// Joins the parts of a row.  All their lists have room in LDS, one behind the other; 256 / parts threads bring a list, eight loads at a time.
template <typename T>
__global__ void __launch_bounds__(kThreads) top_logits_join_kernel(TopShape a) {
    __shared__ TopLds<kJoinRoom> s;
    const uint64_t row = a.row0 + blockIdx.x;
    const uint32_t k = a.k, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    TopShape::Part part{-kInf, 0.f, 0, 0};                        // of lane's part (parts <= 64)
    if (lane < a.parts) part = a.found[row * a.parts + lane];
    Spread spread = wave == 0 ? Spread{part.max, part.sum} : kNoSpread;
    uint32_t upto = part.held;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t other = (uint32_t)__shfl_up((int)upto, o);
        if (lane >= (uint32_t)o) upto += other;
    }
    const uint32_t held = (uint32_t)__shfl((int)upto, 63);
    const uint32_t of_list = kThreads >> (32 - __builtin_clz(a.parts - 1)), p = threadIdx.x / of_list, from = threadIdx.x % of_list;   // (parts > 1)
    const uint32_t n = (uint32_t)__shfl((int)part.held, (int)(p & 63)), to = (uint32_t)__shfl((int)upto, (int)(p & 63)) - n;
    if (p < a.parts) {
        const uint64_t* list = a.lists + (row * a.parts + p) * a.room;
        for (uint32_t q = from; q < n; q += 8 * of_list) {
            uint64_t rank[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) rank[i] = list[q + i * of_list < n ? q + i * of_list : q];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (q + i * of_list < n) s.list[to + q + i * of_list] = rank[i];
        }
    }
    __syncthreads();
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    write_pairs(s, held, k, z, a.pairs + row * k);
    if (!a.lse) return;
    const float scale = kLog2e / a.temperature;
    spread = workgroup_spread<kWaves>(spread, scale, s.sums);
    if (threadIdx.x == 0) a.lse[row] = row_lse(spread, scale, a.temperature);
}

// Workgroups of a row: as many as fill the GPU, each with a stretch or more, and not more than can send k logits each to be joined.
template <typename T>
void top_plan(uint64_t rows, uint64_t vocab, uint32_t k, uint32_t& parts, uint64_t& part_logits, uint32_t& room) {
    constexpr uint64_t stretch = kThreads * kPieces * (16 / sizeof(T));
    const uint64_t stretches = (vocab + stretch - 1) / stretch;
    uint64_t p = rows >= 512 ? 1 : 1024 / rows;
    if (p > stretches) p = stretches;
    if (p > 64) p = 64;
    if (p > kJoinRoom / k) p = kJoinRoom / k;
    if (p < 1) p = 1;
    const uint64_t each = (stretches + p - 1) / p;
    part_logits = each * stretch;
    parts = (uint32_t)((stretches + each - 1) / each);
    room = kJoinRoom / parts < kLong ? kJoinRoom / parts : kLong;
}

template <typename T>
void launch_top_of(const LogitsArgs& args, hipStream_t stream) {
    TopShape a{};
    static_cast<LogitsArgs&>(a) = args;
    top_plan<T>(a.rows, a.vocab, a.k, a.parts, a.part_logits, a.room);
    a.lists = static_cast<uint64_t*>(a.work);
    a.found = reinterpret_cast<TopShape::Part*>(a.lists + a.rows * a.parts * a.room);
    for (uint64_t r = 0; r < a.rows; r += kRowsOfLaunch) {
        a.row0 = r;
        const unsigned here = (unsigned)(a.rows - r < kRowsOfLaunch ? a.rows - r : kRowsOfLaunch);
        hipLaunchKernelGGL(top_logits_kernel<T>, dim3(here, a.parts), dim3(kThreads), 0, stream, a);
        if (a.parts > 1) hipLaunchKernelGGL(top_logits_join_kernel<T>, dim3(here), dim3(kThreads), 0, stream, a);
    }
}

}  // namespace

uint64_t top_logits_work_bytes(const ds_logits& l) {
    uint32_t parts = 1, room = 0;
    uint64_t part_logits;
    by_dtype(l.dtype, [&](auto kind) { top_plan<decltype(kind)>(l.rows, l.vocab, l.k, parts, part_logits, room); });
    return parts > 1 ? l.rows * parts * (room * sizeof(uint64_t) + sizeof(TopShape::Part)) : 0;
}

hipError_t launch_top_logits(const LogitsArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_top_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
