// A token of every row of logits from a given random number (ds_sample).
//
// A row's order (larger first, of equal ones the lower index) is never made.  Every filter keeps a beginning of it, so that all that is needed of a filter is the
// mass of what it keeps, and the token is where the mass passes u times the smallest of these.  Each is one question: at which place of the order do count
// or mass reach a number?  Bins that follow the order answer it but for what lies in one bin, whose logits are then gathered, ranked and summed.
//   Masses exp((z - max) / T) are whole numbers of 2^-bits, made in 64 bits: their sums are exact, so that they depend on no order, may be made with
// atomics, and differ from the formula's by 4e-14 of each mass and half a unit of 2^-bits a logit (bits: 51, and from 2^11 logits on 62 less those of their number: 45 for 131072).  (A token is
// wrong where u comes closer to a border than the sums are off: with sums in 32 bits in one row of ten of 131072 logits.)
//   How a row is gone about, by its type, length and number:
// - up to 512 logits, and in many rows of fp32 and fp16 without a top_k up to 2048, a wave each, the row in LDS (sample_wave_kernel).  Vector instructions bound it: 222 a logit of 500, which
//   keep the vector units busy for 73 % of the clocks;
// - a workgroup each (sample_kernel), which keeps 32 to 128 KB of the row in registers, so that what needs another look at it need not ask memory: passes over a
//   row are bound by what the chip's fabric carries (about 6.6 TB/s), and caches behind it are no faster.  bf16, and rows with a top_k, count logits in fixed bins while they
//   come in.  A bin of bf16 is a number: sums, filters and the token's value are arithmetic on counts, and the last look finds the nth logit of that value.  For a top_k the walk from
//   the largest bin on ends at the k-th's, and what lies above goes into a list that is put in order.  Rows with min_p alone are listed after the first look.  Rows of fp32 and fp16 that
//   need sums of everything make masses of all logits.  In line (up to 32768 logits of many rows) 65 vector instructions a logit, 18 of them the 64-bit exponential's, bound these: 4096 x 32003, fp32,
//   top_p, 322 us, vector units 74 % of the clocks, LDS 23 %, 1.9 readings.  Out of line (answer_any) a row is read 4.6 times, from memory: 4096 x 65536, 762 us for 5.0 GB, 6.5 TB/s;
// - few long rows by several workgroups, four launches (sample_most_kernel and behind it);
// - everything that this leaves open (lists that are too long, ties beyond them, largest logits beyond 4080) by answer_any, at leisure.
//   Calls, us, and what a pass over the logits takes at 6.63 TB/s: 1 x 32000, bf16, k = 50, p = 0.95, 10 (a launch, two trips to memory, twenty barriers); 256 x 32003, fp32, min_p, 13 (4.9);
// 1024 x 131072, bf16, p = 0.95, 84 (40); 2048 x 65536, fp32, k = 100, p = 0.9, 118 (81); 4096 x 131072, bf16, 246 (162).  The last one as two workgroups of 512 threads on a compute unit
// takes 252 us, 63000 clocks a row.  Of these counting takes 27000: an atomic of 64 lanes on LDS takes 9 clocks, 6 of them because lanes meet in banks.  The rest is a chain of
// short phases (masses of bins 6400, the token's place in the row 10000), in which the other workgroup counts, or, of three of 256 threads, as it runs, the other two.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_logits.h"
#include "dsq_sample_bins.h"

namespace dsq {
namespace {

constexpr uint64_t kRowsOfLaunch = 1u << 21;                      // a launch dimension holds fewer than 2^32 work-items
constexpr uint32_t kBins = 2048, kList = 512, kParts = 256;       // bins of a row; logits that are ranked at once; bins of a bin
constexpr uint32_t kAbove = 768, kOctaves = 1024;                 // bins for the logits of the largest one's sign; how far below T they are told apart
constexpr int kPieces = 4;                                        // 16-byte pieces that a thread asks for at a time

struct SampleShape : SampleArgs {
    uint64_t row0;
};

// exp((z - max) / T) of logits as whole numbers of 2^-bits.
struct Masses {
    double max, scale, least;                                     // scale: log2(e) / T; exponents below `least` count as that
    int bits;
    __device__ __forceinline__ uint64_t operator()(float z) const {
        const double x = fmax(((double)z - max) * scale, least);
        const double shifted = x + 0x1.8p52, r = x - (shifted - 0x1.8p52);                 // (its lowest bits are the nearest whole number)
        // 2^r, |r| <= 1/2: the polynomial of degree 9 through 1 that is off by 3.7e-14 at most (interpolation at Chebyshev's points)
        double p = 0x1.b63880e70be2cp-24;
        p = fma(p, r, 0x1.63d136334c4f7p-20);
        p = fma(p, r, 0x1.ffcb95156ef54p-17);
        p = fma(p, r, 0x1.4308ac85ad2d9p-13);
        p = fma(p, r, 0x1.5d87fe86fe961p-10);
        p = fma(p, r, 0x1.3b2ab7181b742p-7);
        p = fma(p, r, 0x1.c6b08d7047e52p-5);
        p = fma(p, r, 0x1.ebfbdff823cedp-3);
        p = fma(p, r, 0x1.62e42fefa39efp-1);
        p = fma(p, r, 1.0);
        const double v = __builtin_ldexp(p, (int)__double_as_longlong(shifted) + bits) + 0x1p52;    // (its lowest 52 bits are the number)
        return (uint64_t)__double_as_longlong(v) & ((1ull << 52) - 1);
    }
};

// A number that is the same in every lane, where it costs no register of each.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ double uniform(double v) {
    const uint64_t bits = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)uniform((uint32_t)(bits >> 32)) << 32 | uniform((uint32_t)bits)));
}

// Bins that follow the order: a logit's is the number that the 15 leading bits of its magnitude make, those below `base` as one, `top` of them above it; what lies
// behind the last one is in it.
struct Bins {
    int32_t base, top;
    uint32_t last;
    __device__ __forceinline__ uint32_t operator()(float z) const {
        const uint32_t bits = __float_as_uint(z);
        int32_t c = (int32_t)(bits >> 16 & 0x7FFFu) - base;
        c = c > 0 ? c : 0;
        const uint32_t bin = (uint32_t)(top - ((int32_t)bits < 0 ? -c : c));
        return bin < last ? bin : last;
    }
    // The largest and the smallest number of a bin.
    __device__ float highest(uint32_t bin) const {
        const int32_t v = top - (int32_t)bin;
        if (v > 0) {
            const uint32_t bits = (uint32_t)(base + v) << 16 | 0xFFFFu;
            return __uint_as_float(bits < 0x7F800000u ? bits : 0x7F800000u);
        }
        return v == 0 ? __uint_as_float((uint32_t)base << 16 | 0xFFFFu) : -__uint_as_float((uint32_t)(base - v) << 16);
    }
    __device__ float lowest(uint32_t bin) const {
        const int32_t v = top - (int32_t)bin;
        if (bin == last) return -kInf;
        if (v > 0) return __uint_as_float((uint32_t)(base + v) << 16);
        const uint32_t bits = (uint32_t)(base - v) << 16 | 0xFFFFu;
        return -__uint_as_float(bits < 0x7F800000u ? bits : 0x7F800000u);
    }
    // The only number of a bin, if logits have 8 bits ...
    __device__ __forceinline__ float number(uint32_t bin) const { return (int32_t)bin < top ? lowest(bin) : highest(bin); }
    // ... and this is true.
    __device__ __forceinline__ bool single(uint32_t bin) const { return bin != (uint32_t)top && bin != last; }
};
// Bins for rows whose largest logit and what matters below it lie between -4080 and 4080, whatever it is: 128 of each power of two from 2^-20 on.  What lies
// beyond is mostly masked and would be one address for many: each lane has a bin of its own for it, 64 at either end.
constexpr int32_t kFixedBase = (127 - 20) << 7, kFixedSide = 4095, kFixedTop = kFixedSide + 63;
constexpr uint32_t kFixedFirst = 63, kFixedLast = kFixedTop + kFixedSide, kFixedCounts = (kFixedLast + 64 + 3) / 4 * 4;
constexpr uint32_t kFixedBins = 8192;                             // from kFixedFirst on: those with an answer in them, and two
constexpr uint32_t kGroups = kFixedBins / 16;
constexpr float kFixedMost = 4080.f;                              // the first number of those
__device__ __forceinline__ Bins fixed_bins() { return {kFixedBase, kFixedTop, kFixedLast}; }
// Bins for any row.
__device__ __forceinline__ Bins bins_of(float max, float temperature) {
    const int32_t m = (int32_t)(__float_as_uint(max) >> 16 & 0x7FFFu), t = (int32_t)(__float_as_uint(temperature) >> 16) - (int32_t)kOctaves;
    Bins b;
    b.base = max < 0.f ? m : m - (int32_t)kAbove;
    if (b.base < t) b.base = t;
    if (b.base < 0) b.base = 0;
    if (b.base > 0x7F7F) b.base = 0x7F7F;
    const int32_t c = m > b.base ? m - b.base : 0;
    b.top = max < 0.f ? -c : c;
    b.last = kBins - 1;
    return b;
}
__device__ __forceinline__ float of_key(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

template <int THREADS>
struct SampleLds {
    union {
        uint32_t count[kFixedCounts];
        struct {
            uint64_t list[kList];                                 // ranks of the logits gathered
            union {
                struct {
                    uint64_t sorted[kList], upto[kList];          // in order; the mass through each
                };
                u32x4 queue[kList];                               // pieces with something to gather, before that
            };
            union {
                struct {
                    uint64_t part_mass[kParts];
                    uint32_t part_count[kParts];
                };
                uint32_t queue_column[kList];                     // of their first logits
            };
            uint64_t mass[kBins];                                 // of bins, and then what lies before them
        };
    };
    uint64_t group[kGroups];                                      // counts or masses of sixteen fixed bins each, and then of all before
    uint64_t sums[THREADS / 64];
    uint32_t counts[THREADS / 64];
    float most[THREADS / 64];
    uint64_t before, through;                                     // answers
    uint32_t held, queued, bin, ahead, least, index;
    float value;
};
// Of a kernel, and of the functions that it calls: one for each, so that it has an address that is known.
template <typename T, int THREADS>
__device__ __forceinline__ SampleLds<THREADS>& sample_lds() {
    __shared__ SampleLds<THREADS> s;
    return s;
}

// a's low (or high) 16 bits times b's, as signed numbers, and c.
template <bool A_HIGH, bool B_HIGH>
__device__ __forceinline__ uint32_t multiply_add_16(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    if constexpr (A_HIGH && B_HIGH) asm("v_mad_i32_i16 %0, %1, %2, %3 op_sel:[1,1,0,0]" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    else if constexpr (A_HIGH) asm("v_mad_i32_i16 %0, %1, %2, %3 op_sel:[1,0,0,0]" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    else asm("v_mad_i32_i16 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// The sum of the lanes up to the own one, by register permutations: one, two, four and eight lanes on in sixteen, then a sixteen's last to the next one's, and that of 32
// to the rest.
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V add_other(V v) {
    if constexpr (sizeof(V) == 8) {
        const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xF, false);
        return v + ((uint64_t)high << 32 | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));
    } else {
        return v + (V)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
    }
}
template <typename V>
__device__ __forceinline__ V upto_lane(V v) {
    v = add_other<0x111, 0xF>(v);                                 // row_shr 1, 2, 4, 8
    v = add_other<0x112, 0xF>(v);
    v = add_other<0x114, 0xF>(v);
    v = add_other<0x118, 0xF>(v);
    v = add_other<0x142, 0xA>(v);                                 // row_bcast 15, 31
    return add_other<0x143, 0xC>(v);
}
__device__ __forceinline__ uint64_t of_lane(uint64_t v, uint32_t lane) {
    return (uint64_t)__builtin_amdgcn_readlane((uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)v, lane);
}

__device__ __forceinline__ void wave_sync() {                     // what lanes wrote to LDS before is read by others after
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// What lies before the thread's v in the workgroup, and all of it.
template <int THREADS, typename V>
__device__ __forceinline__ V before_thread(V v, V* sums, V& all) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const V upto = upto_lane(v);
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    V before = 0;
    all = 0;
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 64; ++w) {
        const V of = sums[w];
        before += w < wave ? of : 0;
        all += of;
    }
    return before + upto - v;
}

// The column of the nth (from 1) logit that equals `value`: each wave counts those of a stretch of the row.
template <typename T, int THREADS>
__device__ __attribute__((noinline)) void find_nth(const T* z, uint32_t vocab, float value, uint64_t nth) {
    constexpr uint32_t E = Pieces<T>::E;
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    constexpr uint32_t kStep = 64 * E;
    const uint32_t stretch = ((vocab + THREADS / 64 - 1) / (THREADS / 64) + kStep - 1) / kStep * kStep;
    const uint64_t begin = (uint64_t)wave * stretch;
    const uint32_t from = begin < vocab ? (uint32_t)begin : vocab, to = vocab - from < stretch ? vocab : from + stretch;
    auto equal = [&](uint32_t at) {                           // bits of the lane's elements that are it
        uint32_t bits = 0;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
            if (at + e < to && (float)z[at + e] == value) bits |= 1u << e;
        return bits;
    };
    uint32_t mine = 0, all;
    for (uint32_t at = from + lane * E; at < to; at += kStep) mine += (uint32_t)__popc(equal(at));
    uint64_t before = before_thread<THREADS>(mine, s.counts, all);
    before = (uint64_t)(uint32_t)__shfl((int)before, 0);      // of the wave
    const uint32_t of_wave = s.counts[wave];
    if (nth <= before || nth > before + of_wave) {
        __syncthreads();
        return;
    }
    uint64_t left = nth - before;
    for (uint32_t base = from; base < to; base += kStep) {
        const uint32_t at = base + lane * E, bits = at < to ? equal(at) : 0;
        uint32_t upto = (uint32_t)__popc(bits);
        const uint32_t own = upto;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t other = (uint32_t)__shfl_up((int)upto, o);
            if (lane >= (uint32_t)o) upto += other;
        }
        const uint32_t total = (uint32_t)__shfl((int)upto, 63);
        if (left > total) {
            left -= total;
            continue;
        }
        if (left <= upto && left > upto - own) {
            uint32_t rest = bits;
            for (uint64_t i = left - (upto - own); i > 1; --i) rest &= rest - 1;
            s.index = at + (uint32_t)__builtin_ctz(rest);
        }
        break;
    }
    __syncthreads();
}

// A row of which the thread keeps N 16-byte pieces in registers between the passes; what does not fit comes from memory, or its caches, again, the last of it
// first: it is the likeliest to be there.
template <typename T, int THREADS, int N>
struct Kept {
    static constexpr bool kNumbers = std::is_same_v<T, __bf16>;
    static constexpr uint32_t E = Pieces<T>::E, kHeld = N * THREADS;                       // pieces of a row that are held
    using Piece = typename Pieces<T>::Piece;
    const T* z;
    uint32_t vocab, whole;                                        // whole: pieces without the ragged end
    u32x4 held[N];
    T last;                                                       // of the ragged end

    __device__ __forceinline__ u32x4 load(uint32_t piece) const { return __builtin_bit_cast(u32x4, *reinterpret_cast<const Piece*>(z + piece * E)); }
    static constexpr uint32_t kNothing = sizeof(T) == 4 ? 0xFF800000u : kNumbers ? 0xFF80FF80u : 0xFC00FC00u;             // minus infinity
    __device__ __forceinline__ static u32x4 nothing() { return u32x4{kNothing, kNothing, kNothing, kNothing}; }
    __device__ __forceinline__ Kept(const T* row, uint32_t length) : z(row), vocab(length), whole(length / E) {
#pragma unroll
        for (int p = 0; p < N; ++p) {
            held[p] = nothing();
            if (p * THREADS + threadIdx.x < whole) held[p] = load(p * THREADS + threadIdx.x);
        }
        last = whole * E + threadIdx.x < vocab ? z[whole * E + threadIdx.x] : (T)-kInf;
    }
    __device__ __forceinline__ uint32_t last_column() const { return whole * E + threadIdx.x; }
    // f(piece, its first column) for what is held ...
    template <typename F>
    __device__ __forceinline__ void of_held(F f) const {
#pragma unroll
        for (int p = 0; p < N; ++p)
            if (p * THREADS < whole) f(held[p], (p * THREADS + threadIdx.x) * E);
    }
    // ... and for stretch i of what is not
    static constexpr uint32_t kStretch = kPieces * THREADS;
    __device__ __forceinline__ uint32_t stretches() const { return whole > kHeld ? (whole - kHeld + kStretch - 1) / kStretch : 0; }
    __device__ __forceinline__ void fetch(u32x4 (&raw)[kPieces], uint32_t i) const {
        const uint32_t first = kHeld + i * kStretch + threadIdx.x;
        if (kHeld + (i + 1) * kStretch <= whole) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) raw[p] = load(first + p * THREADS);
        } else {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                raw[p] = nothing();
                if (first + p * THREADS < whole) raw[p] = load(first + p * THREADS);
            }
        }
    }
    __device__ __forceinline__ static uint32_t column(uint32_t i, int p) { return (kHeld + i * kStretch + p * THREADS + threadIdx.x) * E; }

    __device__ __forceinline__ static void values(u32x4 raw, float (&v)[E]) {
        const Piece piece = __builtin_bit_cast(Piece, raw);
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) v[e] = (float)piece[e];
    }
    // The thread's largest logit.
    __device__ __forceinline__ float largest() const {
        float max = (float)last;
        auto f = [&](u32x4 raw, uint32_t) {
            float v[E];
            values(raw, v);
            max = max_or_nan(max, largest_of(v));
        };
        of_held(f);
        for (uint32_t i = 0, n = stretches(); i < n; ++i) {
            u32x4 raw[kPieces];
            fetch(raw, i);
#pragma unroll
            for (int p = 0; p < kPieces; ++p) f(raw[p], 0);
        }
        return max;
    }
    // Counts logits in fixed bins; with places as multiples of a sign's step added to the middle, eight vector instructions for two bf16 logits (twelve, with two's complements and the least place of
    // each thread kept: 4096 x 131072 268 us, so 263).  Returns the thread's largest one; of bf16, whose bins tell it, whether it met a NaN.
    struct Counted {
        float max;
        bool nan;
    };
    __device__ __forceinline__ Counted count_fixed() const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        auto add = [&](uint32_t place) { atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(s.count) + place), 1u); };
        const uint32_t most = kFixedSide + (threadIdx.x & 63), top = 4 * kFixedTop;        // (places are in bytes)
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 magnitudes = 0;
        float max = -kInf;
        const float least_magnitude = __uint_as_float((uint32_t)kFixedBase << 16), most_magnitude = __uint_as_float((kFixedBase + most) << 16);
        auto f = [&](u32x4 raw) {
            if constexpr (kNumbers) {                             // two at a time
                const u16x2 base = (uint16_t)kFixedBase, side = (uint16_t)most;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t bits = raw[i];                 // (a cast of the element itself would be one of the first)
                    const u16x2 magnitude = __builtin_bit_cast(u16x2, bits & 0x7FFF7FFFu);
                    magnitudes = __builtin_elementwise_max(magnitudes, magnitude);
                    const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_elementwise_sub_sat(magnitude, base), side));
                    const uint32_t step = __builtin_bit_cast(uint32_t, (u16x2)((__builtin_bit_cast(u16x2, bits) >> (uint16_t)15) * (uint16_t)8 + (uint16_t)-4));
                    add(multiply_add_16<false, false>(c, step, top));                      // top - 4 c, or top + 4 c where the sign is set
                    add(multiply_add_16<true, true>(c, step, top));
                }
            } else {
                float v[E];
                values(raw, v);
                max = max_or_nan(max, largest_of(v));
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) {
                    const uint32_t magnitude = __float_as_uint(__builtin_amdgcn_fmed3f(fabsf(v[e]), least_magnitude, most_magnitude));
                    const uint32_t step = (__float_as_uint(v[e]) >> 31) * 8 - 4;
                    add(multiply_add_16<true, false>(magnitude - ((uint32_t)kFixedBase << 16), step, top));
                }
            }
        };
        const uint32_t n = stretches();
        u32x4 ahead[kPieces];                                     // (a stretch is on its way while what comes before it is counted: 4096 x 131072, bf16, 263 us, so 258)
        if (n) fetch(ahead, 0);
        of_held([&](u32x4 raw, uint32_t) { f(raw); });
        for (uint32_t i = 0; i < n; ++i) {
            u32x4 raw[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) raw[p] = ahead[p];
            if (i + 1 < n) fetch(ahead, i + 1);
#pragma unroll
            for (int p = 0; p < kPieces; ++p) f(raw[p]);
        }
        if (whole * E < vocab) {
            u32x4 end = nothing();
            if constexpr (sizeof(T) == 4) end[0] = __builtin_bit_cast(uint32_t, last);
            else end[0] = (end[0] & 0xFFFF0000u) | __builtin_bit_cast(uint16_t, last);
            f(end);
        }
        return {max, magnitudes[0] > 0x7F80 || magnitudes[1] > 0x7F80};
    }
    // f(logit) for all of them.
    template <typename F>
    __device__ __forceinline__ void of_all(F f) const {
        auto piece = [&](u32x4 raw) {
            float v[E];
            values(raw, v);
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) f(v[e]);
        };
        of_held([&](u32x4 raw, uint32_t) { piece(raw); });
        for (uint32_t i = stretches(); i-- > 0;) {
            u32x4 raw[kPieces];
            fetch(raw, i);
#pragma unroll
            for (int p = 0; p < kPieces; ++p) piece(raw[p]);
        }
        f((float)last);
    }
    // What is rare is looked for in two steps, so that the code for each piece is short: pieces with some of it, by test(piece), go into a queue (queue, for M of them), and
    // is(logit) tells for the queue's logits from piece `from` on which ones go to add(logit, column) (expand).
    __device__ __forceinline__ void clear_queue() const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        __syncthreads();
        if (threadIdx.x == 0) s.held = s.queued = 0;
        __syncthreads();
    }
    template <int M, typename F, typename C>
    __device__ __forceinline__ void queue(const u32x4 (&raw)[M], C column_of, F test) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        uint32_t mask = 0;
#pragma unroll
        for (int p = 0; p < M; ++p) mask |= test(raw[p]) ? 1u << p : 0u;
        if (!__ballot(mask != 0)) return;
        const uint32_t mine = (uint32_t)__popc(mask), upto = upto_lane(mine), all = (uint32_t)__builtin_amdgcn_readlane(upto, 63);
        uint32_t place = 0;
        if ((threadIdx.x & 63) == 0) place = atomicAdd(&s.queued, all);
        place = uniform(place) + upto - mine;
#pragma unroll
        for (int p = 0; p < M; ++p)
            if (mask >> p & 1u) {
                if (place < kList) {
                    s.queue[place] = raw[p];
                    s.queue_column[place] = column_of(p);
                }
                ++place;
            }
    }
    template <typename F, typename A>
    __device__ __forceinline__ uint32_t expand(uint32_t from, F is, A add) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        __syncthreads();
        const uint32_t queued = s.queued;
        if (queued <= kList)
            for (uint32_t i = from * E + threadIdx.x; i < queued * E; i += THREADS) {
                const float v = (float)reinterpret_cast<const T*>(&s.queue[i / E])[i % E];
                if (is(v)) add(v, s.queue_column[i / E] + i % E);
            }
        __syncthreads();
        return queued;
    }
    // Gathers logits as ranks, those from lo to hi or those of which is(logit) is true; returns how many there are, or more than kList.
    __device__ __forceinline__ uint32_t gather(float lo, float hi) const {
        return gather_if([&](u32x4 raw) {
            float v[E];
            values(raw, v);
            return largest_of(v) >= lo;
        }, [&](float v) { return v >= lo && v <= hi; });
    }
    template <typename F>
    __device__ __forceinline__ uint32_t gather_those(F is) const {
        return gather_if([&](u32x4 raw) {
            float v[E];
            values(raw, v);
            bool some = false;
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) some |= is(v[e]);
            return some;
        }, is);
    }
    template <typename S, typename F>
    __device__ __forceinline__ uint32_t gather_if(S test, F is) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        clear_queue();
        auto add = [&](float v, uint32_t column) {
            const uint32_t place = atomicAdd(&s.held, 1u);
            if (place < kList) s.list[place] = logit_rank(v, column);
        };
        queue(held, [&](int p) { return (p * THREADS + threadIdx.x) * E; }, test);
        for (uint32_t i = stretches(); i-- > 0;) {
            u32x4 raw[kPieces];
            fetch(raw, i);
            queue(raw, [&](int p) { return column(i, p); }, test);
        }
        if (whole * E < vocab && is((float)last)) add((float)last, last_column());
        const uint32_t queued = expand(0, is, add);
        return queued <= kList ? s.held : queued;
    }
    // The column of the nth (from 1) of the n logits, of bf16, that equal `value`: from the front among those held, or from the row's end.
    __device__ __forceinline__ void find(float value, uint64_t nth, uint32_t n) const {
        static_assert(kNumbers);
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        // equal numbers are equal bits, but for the sign of 0
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        const uint32_t keep = value == 0.f ? 0x7FFF7FFFu : ~0u, bits = __builtin_bit_cast(uint16_t, (T)value) * 0x10001u & keep;
        auto test = [&](u32x4 raw) {
            u32x4 d;
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = (raw[i] & keep) ^ bits;
            auto least = [](uint32_t x, uint32_t y) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y))); };
            const uint32_t m = least(least(d[0], d[1]), least(d[2], d[3]));
            return (m & 0xFFFFu) == 0 || m < 0x10000u;
        };
        auto is = [&](float v) { return v == value; };
        auto add = [&](float, uint32_t column) {
            const uint32_t place = atomicAdd(&s.held, 1u);
            if (place < kList) s.list[place] = column;
        };
        const uint32_t rest = stretches();
        clear_queue();
        queue(held, [&](int p) { return (p * THREADS + threadIdx.x) * E; }, test);
        auto end = [&] {
            if (whole * E < vocab && is((float)last)) add(0.f, last_column());
        };
        if (!rest) end();
        uint32_t queued = expand(0, is, add), found = s.held;
        bool forward = true;
        if (rest && queued <= kList && nth > found) {
            forward = false;
            nth = n - nth + 1;
            clear_queue();
            end();
            queued = 0;
            for (uint32_t i = rest; i-- > 0;) {
                u32x4 raw[kPieces];
                fetch(raw, i);
                queue(raw, [&](int p) { return column(i, p); }, test);
                queued = expand(queued, is, add);
                found = s.held;
                if (found >= nth || queued > kList) break;
            }
        }
        if (queued > kList || found > kList) return find_nth<T, THREADS>(z, vocab, value, forward ? nth : n - nth + 1);
        for (uint32_t i = threadIdx.x; i < found; i += THREADS) {
            const uint64_t mine = s.list[i];
            uint32_t place = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < found; ++j) place += (s.list[j] < mine) == forward ? 1u : 0u;
            if (place == (forward ? nth - 1 : nth)) s.index = (uint32_t)mine;              // (backwards it counts itself)
        }
        __syncthreads();
    }
};

enum Question { kCount, kMass, kValue };                          // at which place do count or mass reach a number, or logits a value

// Puts s.list's n ranks (n <= kList) in order into s.sorted: each goes where as many are above it.  Of few, four threads count for each.  (Numbers that go
// to all lanes from a register by v_readlane instead of from LDS: 64 x 30000, k = 400, 24 us, and 17.)
template <typename T, int THREADS>
__device__ __forceinline__ void sort_list(uint32_t n) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    if (n * 4 <= THREADS) {
        const uint32_t i = threadIdx.x / 4;
        const uint64_t mine = i < n ? s.list[i] : 0;
        uint32_t place = 0;
#pragma unroll 4
        for (uint32_t j = threadIdx.x & 3; j < n; j += 4) place += s.list[j] > mine ? 1u : 0u;
        place = over_lanes<4>(place, [](uint32_t x, uint32_t y) { return x + y; });
        if (i < n && (threadIdx.x & 3) == 0) s.sorted[place] = mine;
    } else {
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t mine = s.list[i];
            uint32_t place = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < n; ++j) place += s.list[j] > mine ? 1u : 0u;
            s.sorted[place] = mine;
        }
    }
    __syncthreads();
}

template <typename T, int THREADS>
struct Row {
    static constexpr bool kNumbers = std::is_same_v<T, __bf16>;   // a bin is a number
    static constexpr uint32_t E = Pieces<T>::E;
    using Piece = typename Pieces<T>::Piece;
    const T* z;
    uint32_t vocab;
    Masses masses;
    float least;                                                  // logits below it have no mass

    // f(values, column of the first) for all 16-byte pieces; what lies behind the end is minus infinity.
    template <typename F>
    __device__ __forceinline__ void stream(F f) const {
        uint32_t at = threadIdx.x * E;
        for (; at + (kPieces - 1) * THREADS * E + E <= vocab; at += kPieces * THREADS * E) {
            Piece raw[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) raw[p] = *reinterpret_cast<const Piece*>(z + at + p * THREADS * E);
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                float v[E];
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) v[e] = (float)raw[p][e];
                f(v, at + p * THREADS * E);
            }
        }
        for (; at < vocab; at += THREADS * E) {
            float v[E];
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) v[e] = at + e < vocab ? (float)z[at + e] : -kInf;
            f(v, at);
        }
    }

    __device__ __forceinline__ uint32_t fixed_count(uint32_t bin) const { return bin < kFixedLast ? sample_lds<T, THREADS>().count[bin] : 0; }
    // The first fixed bin with a logit in it, which each wave looks for by itself, eight powers of two at a time.
    __device__ __forceinline__ uint32_t first_bin() const {
        const u32x4* const four = reinterpret_cast<const u32x4*>(sample_lds<T, THREADS>().count);
        constexpr uint32_t kFours = kFixedCounts / 4, kAtOnce = 4;
#pragma unroll 1
        for (uint32_t from = 0; from < kFours; from += 64 * kAtOnce) {
            u32x4 n[kAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t at = from + i * 64 + (threadIdx.x & 63);
                n[i] = at < kFours ? four[at] : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint64_t some = __ballot((n[i][0] | n[i][1] | n[i][2] | n[i][3]) != 0);
                if (!some) continue;
                const uint32_t lane = (uint32_t)__builtin_ctzll(some), mine = n[i][0] ? 0u : n[i][1] ? 1u : n[i][2] ? 2u : 3u;
                return uniform((from + i * 64 + lane) * 4 + (uint32_t)__builtin_amdgcn_readlane(mine, lane));
            }
        }
        return kFixedLast;
    }
    // s.group, which is cleared: what of(bin, its count) gives for sixteen bins.
    template <typename F>
    __device__ __forceinline__ void sum_groups(F of) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        constexpr uint32_t kOwn = kFixedBins / THREADS, kAtOnce = 16;
#pragma unroll 1
        for (uint32_t from = 0; from < kOwn; from += kAtOnce) {
            uint32_t n[kAtOnce];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) n[i] = fixed_count(kFixedFirst + (from + i) * THREADS + threadIdx.x);
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i)
                if (n[i]) {
                    const uint32_t at = (from + i) * THREADS + threadIdx.x;
                    atomicAdd(reinterpret_cast<unsigned long long*>(&s.group[at / 16]), (unsigned long long)of(kFixedFirst + at, n[i]));
                }
        }
        __syncthreads();
    }
    // In the first wave: what lies before each of the groups takes their place.  Returns the sum of all.
    __device__ __forceinline__ uint64_t sum_before_groups() const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        constexpr uint32_t kEach = kGroups / 64;
        uint64_t own[kEach], sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            own[i] = s.group[threadIdx.x * kEach + i];
            sum += own[i];
        }
        const uint64_t upto = upto_lane(sum), all = of_lane(upto, 63);
        uint64_t before = upto - sum;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            s.group[threadIdx.x * kEach + i] = before;
            before += own[i];
        }
        wave_sync();
        return all;
    }
    __device__ __forceinline__ void clear_groups() const {
        for (uint32_t i = threadIdx.x; i < kGroups; i += THREADS) sample_lds<T, THREADS>().group[i] = 0;
    }
    // In a wave: the bin in which the sum reaches t (1 <= t <= all), or `bin` itself, what of(bin, count) gives for it and what lies before it.
    struct FoundBin {
        uint32_t bin;
        uint64_t here, before;
    };
    template <typename F>
    __device__ __forceinline__ FoundBin find_bin(bool given, uint32_t bin, uint64_t t, F of) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        const uint32_t lane = threadIdx.x & 63;
        uint32_t group;
        if (given) {
            group = (bin - kFixedFirst) / 16;
        } else {
            group = 0;
#pragma unroll
            for (uint32_t i = 0; i < kGroups; i += 64) group += (uint32_t)__popcll(__ballot(s.group[i + lane] < t));
            --group;                                              // (the first group has nothing before it)
        }
        const uint32_t mine = kFixedFirst + group * 16 + (lane & 15), n = fixed_count(mine);
        const uint64_t here = n ? of(mine, n) : 0, ahead = s.group[group];
        uint64_t upto = add_other<0x111, 0xF>(here);              // (each sixteen lanes by themselves)
        upto = add_other<0x112, 0xF>(upto);
        upto = add_other<0x114, 0xF>(upto);
        upto = add_other<0x118, 0xF>(upto);
        upto += ahead;
        const uint32_t at = uniform(given ? (bin - kFixedFirst) % 16 : (uint32_t)__builtin_ctzll(__ballot(upto >= t)));
        return {kFixedFirst + group * 16 + at, of_lane(here, at), of_lane(upto - here, at)};
    }

    // Gathers the logits from lo to hi (kList of them at most) as ranks; returns how many there are.
    __device__ __forceinline__ uint32_t gather(float lo, float hi) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        __syncthreads();
        if (threadIdx.x == 0) s.held = 0;
        __syncthreads();
        stream([&](const float(&v)[E], uint32_t at) {
            if (!(largest_of(v) >= lo)) return;
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (v[e] >= lo && v[e] <= hi && at + e < vocab) {
                    const uint32_t place = atomicAdd(&s.held, 1u);
                    if (place < kList) s.list[place] = logit_rank(v[e], at + e);
                }
        });
        __syncthreads();
        return s.held;
    }
    // Puts the n gathered logits in order, with the mass through each of them, `before` included.
    __device__ void settle(uint32_t n, uint64_t before) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        sort_list<T, THREADS>(n);
        constexpr uint32_t kEach = kList / THREADS;
        uint64_t mass[kEach], sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t at = threadIdx.x * kEach + i;
            mass[i] = at < n ? masses(of_key((uint32_t)(s.sorted[at] >> 32))) : 0;
            sum += mass[i];
        }
        uint64_t all;
        uint64_t upto = before + before_thread<THREADS>(sum, s.sums, all);
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            upto += mass[i];
            if (threadIdx.x * kEach + i < n) s.upto[threadIdx.x * kEach + i] = upto;
        }
        __syncthreads();
    }
    // Mass through the place in the list where mass reaches t; its index goes to s.index.
    __device__ uint64_t list_mass(uint32_t n, uint64_t before, uint64_t t) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t here = s.upto[i];
            if (here >= t && (i ? s.upto[i - 1] : before) < t) {
                s.through = here;
                s.index = (uint32_t)~s.sorted[i];
            }
        }
        __syncthreads();
        const uint64_t through = s.through;
        __syncthreads();
        return through;
    }
    // Mass through the last logit of the list with z - max >= d.
    __device__ uint64_t list_value(uint32_t n, uint64_t before, double d) const {
        SampleLds<THREADS>& s = sample_lds<T, THREADS>();
        if (threadIdx.x == 0) s.through = before;
        __syncthreads();
        auto kept = [&](uint32_t i) { return (double)of_key((uint32_t)(s.sorted[i] >> 32)) - masses.max >= d; };
        for (uint32_t i = threadIdx.x; i < n; i += THREADS)
            if (kept(i) && (i + 1 == n || !kept(i + 1))) s.through = s.upto[i];
        __syncthreads();
        const uint64_t through = s.through;
        __syncthreads();
        return through;
    }

    // Logits that are all `value`, n of them (kValue), behind `before`.
    __device__ uint64_t among_equals(Question q, float value, uint64_t n, uint64_t before, uint64_t t, double d, bool pick) const {
        const uint64_t mass = masses(value);
        if (q == kValue) return before + ((double)value - masses.max >= d ? n * mass : 0);
        const uint64_t nth = q == kCount ? t : (t - before + mass - 1) / mass;
        if (pick) find_nth<T, THREADS>(z, vocab, value, nth);
        return before + nth * mass;
    }
};

// The answer among the logits from lo to hi: the mass through the place where their count (kCount) or the mass, that of logits before them
// included (kMass), reaches t, or through the last with z - max >= d (kValue).
template <typename T, int THREADS>
__device__ __attribute__((noinline)) uint64_t through(Row<T, THREADS> r, Question q, float lo, float hi, uint64_t before, uint64_t t, double d, bool pick) {
    constexpr uint32_t E = Pieces<T>::E;
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    for (;;) {
        const uint32_t n = r.gather(lo, hi);
        if (q == kCount && t > n) t = n;                      // (what is below `least` was counted, too)
        if (n == 0) return before;
        if (n <= kList) {
            r.settle(n, before);
            if (q == kValue) return r.list_value(n, before, d);
            if (q == kMass) return r.list_mass(n, before, t);
            return s.upto[t - 1];
        }
        if (lo == hi) return r.among_equals(q, lo, n, before, t, d, pick);
        // too many: bins of their own
        const uint32_t first = logit_key(hi), last = logit_key(lo);
        int shift = 0;
        while ((first - last) >> shift >= kParts) ++shift;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < kParts; i += THREADS) {
            s.part_mass[i] = 0;
            s.part_count[i] = 0;
        }
        __syncthreads();
        r.stream([&](const float(&v)[E], uint32_t at) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (v[e] >= lo && v[e] <= hi && at + e < r.vocab) {
                    const uint32_t part = (first - logit_key(v[e])) >> shift;
                    atomicAdd(&s.part_count[part], 1u);
                    atomicAdd(reinterpret_cast<unsigned long long*>(&s.part_mass[part]), (unsigned long long)r.masses(v[e]));
                }
        });
        __syncthreads();
        const uint64_t mass = threadIdx.x < kParts ? s.part_mass[threadIdx.x] : 0;
        const uint32_t count = threadIdx.x < kParts ? s.part_count[threadIdx.x] : 0;
        uint64_t all_mass;
        uint32_t all_count;
        const uint64_t mass_before = before + before_thread<THREADS>(mass, s.sums, all_mass);
        const uint32_t ahead = before_thread<THREADS>(count, s.counts, all_count);
        bool here;
        if (q == kCount) here = ahead < t && t <= (uint64_t)ahead + count;
        else if (q == kMass) here = mass_before < t && t <= mass_before + mass;
        else {
            float border = (float)(r.masses.max + d);
            border = border > hi ? hi : border < lo ? lo : border;
            here = threadIdx.x == (first - logit_key(border)) >> shift;
        }
        if (here) {
            s.bin = threadIdx.x;
            s.before = mass_before;
            s.ahead = ahead;
        }
        __syncthreads();
        const uint32_t high = first - (s.bin << shift), low = high - ((1u << shift) - 1);
        hi = of_key(high == 0x7FFFFFFFu ? high - 1 : high);   // (-0 has the key of +0, which is above)
        lo = high - last < (1u << shift) ? of_key(last) : of_key(low);
        before = s.before;
        if (q == kCount) t -= s.ahead;
        __syncthreads();
    }
}

// What a row is asked for.
struct Asked {
    float temperature, top_p, max;
    uint32_t k;                                                   // 0: all
    uint64_t u;                                                   // times 2^64
    bool by_mass, by_value, infinite;
    double border;                                                // of z - max: by_value
    // what the first logits must reach for top_p of a sum
    __device__ __forceinline__ uint64_t share(uint64_t sum) const {
        if (!(top_p > 0.f)) return 1;
        const uint64_t p = (uint64_t)((double)top_p * 0x1p64), t = __umul64hi(p, sum) + (p * sum ? 1 : 0);
        return t ? t : 1;
    }
};
__device__ __forceinline__ Asked asked_of(const SampleShape& a, uint64_t row) {
    Asked q{};
    q.temperature = a.each.temperature_dev ? a.each.temperature_dev[row] : a.temperature;
    q.top_p = a.each.top_p_dev ? a.each.top_p_dev[row] : a.top_p;
    const int32_t top_k = a.each.top_k_dev ? a.each.top_k_dev[row] : a.top_k;
    q.k = top_k > 0 && (uint64_t)top_k < a.vocab ? (uint32_t)top_k : 0;
    if (!(q.temperature >= __FLT_MIN__ && q.temperature < kInf)) {                         // the largest logit
        q.temperature = 1.f;
        q.k = 1;
    }
    q.by_mass = q.top_p < 1.f;
    return q;
}
// What depends on the row's largest logit, which is a number or plus infinity.
__device__ __forceinline__ void ask(const SampleShape& a, float max, float u, float min_p, Asked& q, Masses& masses, float& least) {
    const double t = (double)q.temperature;
    q.max = max;
    q.infinite = max == kInf;
    q.by_value = min_p > 0.f && !q.infinite;                      // (infinite ones are alike)
    q.border = q.by_value ? t * log((double)(min_p < 1.f ? min_p : 1.f)) : -kInf;
    q.u = !(u > 0.f) ? 0 : u >= 1.f ? ~0ull : (uint64_t)((double)u * 0x1p64);
    masses.max = (double)max;
    masses.scale = uniform(1.44269504088896340736 / t);
    masses.least = q.infinite ? 0.0 : -1000.0;
    masses.bits = 62 - (a.vocab > 1 ? 64 - __builtin_clzll(a.vocab - 1) : 0);
    if (masses.bits > 51) masses.bits = 51;
    // below: masses of less than half of a unit.  (In 32 bits: off by less than what one unit more of the exponent allows for.)
    least = q.infinite ? kInf : fmaxf((float)((double)max - (masses.bits + 2) * 0.69314718055994530942 * t - fabs((double)max) * 0x1p-20), -__FLT_MAX__);
}
__device__ __forceinline__ void no_answer(const SampleShape& a, uint64_t row, float max) {
    a.token[row] = -1;
    if (a.logp) a.logp[row] = max;
}
__device__ __forceinline__ void write_answer(const SampleShape& a, uint64_t row, const Asked& q, const Masses& masses, uint32_t index, float z, uint64_t sum) {
    a.token[row] = (int32_t)index;
    const double y = q.infinite ? 0.0 : ((double)z - (double)q.max) / (double)q.temperature + 0.0;   // (-0 beside +0: not -0, whichever is taken for the largest)
    if (a.logp) a.logp[row] = (float)(y - log(ldexp((double)sum, -masses.bits)));
}

// The mass that is kept, and s.index, out of a list of everything that matters.
template <typename T, int THREADS>
__device__ __forceinline__ uint64_t answer_from_list(const Row<T, THREADS>& r, const Asked& a, uint32_t n) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    r.settle(n, 0);
    uint64_t sum = s.upto[a.k && a.k < n ? a.k - 1 : n - 1];
    if (a.by_mass) sum = r.list_mass(n, 0, a.share(sum));
    if (a.by_value) {
        const uint64_t kept = r.list_value(n, 0, a.border);
        sum = kept < sum ? kept : sum;
    }
    (void)r.list_mass(n, 0, __umul64hi(a.u, sum) + 1);
    return sum;
}

// The same, and the answer written: the workgroup puts the list in order, its first wave does the rest.
template <typename T, int THREADS>
__device__ __forceinline__ void finish_from_list(const SampleShape& shape, uint64_t row, const Row<T, THREADS>& r, const Asked& a, uint32_t n) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    sort_list<T, THREADS>(n);
    if (threadIdx.x >= 64) return;
    const uint32_t each = (n + 63) / 64, first = threadIdx.x * each;                       // in their order: `each` of a lane
    uint64_t sum = 0;
    for (uint32_t i = first; i < first + each && i < n; ++i) {
        sum += r.masses(of_key((uint32_t)(s.sorted[i] >> 32)));
        s.upto[i] = sum;
    }
    const uint64_t before = upto_lane(sum) - sum;
    for (uint32_t i = first; i < first + each && i < n; ++i) s.upto[i] += before;
    wave_sync();
    // places at which f is true, which are the first ones
    auto places = [&](auto f) {
        uint32_t all = 0;
        for (uint32_t i = 0; i < n; i += 64) all += (uint32_t)__popcll(__ballot(i + threadIdx.x < n && f(i + threadIdx.x)));
        return all;
    };
    auto reached = [&](uint64_t t) { return places([&](uint32_t i) { return s.upto[i] < t; }); };
    sum = s.upto[a.k && a.k < n ? a.k - 1 : n - 1];
    if (a.by_mass) sum = s.upto[reached(a.share(sum))];
    if (a.by_value) {
        const uint64_t kept = s.upto[places([&](uint32_t i) { return (double)of_key((uint32_t)(s.sorted[i] >> 32)) - r.masses.max >= a.border; }) - 1];
        sum = kept < sum ? kept : sum;
    }
    const uint64_t token = s.sorted[reached(__umul64hi(a.u, sum) + 1)];
    if (threadIdx.x == 0) write_answer(shape, row, a, r.masses, ~(uint32_t)token, of_key((uint32_t)(token >> 32)), sum);
}

// The bin of the k-th logit (s.bin), the logits before it (s.ahead) and up to its end (s.held): the thread's bins begin with `first` and have `own` logits, and
// there are `before` before them; count(bin).
template <typename T, int THREADS, typename C>
__device__ __forceinline__ void find_kth(uint32_t k, uint32_t before, uint32_t own, uint32_t first, C count) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    if (before < k && k <= before + own) {
        uint32_t upto = before;
        for (uint32_t i = first;; ++i) {
            const uint32_t here = count(i);
            if (k <= upto + here) {
                s.bin = i;
                s.ahead = upto;
                s.held = upto + here;
                break;
            }
            upto += here;
        }
    }
    __syncthreads();
}

// Any row: bins of its own hold masses, and what lies in one of them is gathered.  k_low, k_high: the numbers of the bin of the k-th logit, if k > 0, and k_left the
// how-manieth of it that is, 0 where this is not known yet.
template <typename T, int THREADS>
__device__ __attribute__((noinline)) uint64_t answer_any(Row<T, THREADS> r, float temperature, float top_p, float max, uint32_t k, uint64_t u, double border,
                                                           float k_low, float k_high, uint32_t k_left) {
    Asked a{temperature, top_p, max, k, u, top_p < 1.f, border != -kInf, max == kInf, border};
    constexpr uint32_t E = Pieces<T>::E, kOwn = kBins / THREADS;
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    const Bins bins = bins_of(a.max, a.temperature);
    __syncthreads();
    if (a.k && !k_left) {
        for (uint32_t i = threadIdx.x; i < kBins; i += THREADS) s.count[i] = 0;
        __syncthreads();
        r.stream([&](const float(&v)[E], uint32_t) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (v[e] >= r.least) atomicAdd(&s.count[bins(v[e])], 1u);
        });
        __syncthreads();
        uint32_t own = 0, all;
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) own += s.count[threadIdx.x * kOwn + i];
        const uint32_t before = before_thread<THREADS>(own, s.counts, all);
        if (a.k >= all) a.k = 0;
        if (a.k) {
            find_kth<T, THREADS>(a.k, before, own, threadIdx.x * kOwn, [&](uint32_t i) { return s.count[i]; });
            const uint32_t bin = s.bin, upto = s.held;
            k_left = a.k - s.ahead;
            k_low = bins.lowest(bin);
            k_high = bins.highest(bin);
            if (k_low > r.least) r.least = k_low;
            __syncthreads();
            if (upto <= kList) return answer_from_list(r, a, r.gather(r.least, kInf));
        }
    }
    if (a.k && k_low > r.least) r.least = k_low;
    for (uint32_t i = threadIdx.x; i < kBins; i += THREADS) s.mass[i] = 0;
    __syncthreads();
    uint64_t above = 0;                                           // mass before the k-th's bin
    r.stream([&](const float(&v)[E], uint32_t) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
            if (v[e] >= r.least) {
                const uint64_t mass = r.masses(v[e]);
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[bins(v[e])]), (unsigned long long)mass);
                if (a.k && v[e] > k_high) above += mass;
            }
    });
    __syncthreads();
    uint64_t own = 0, sum;
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i) own += s.mass[threadIdx.x * kOwn + i];
    const uint64_t before = before_thread<THREADS>(own, s.sums, sum);
    if (a.k) {
        (void)before_thread<THREADS>(above, s.sums, above);
        sum = through(r, kCount, r.least, k_high, above, k_left, 0.0, false);
    }
    // the bin in which mass reaches t, or the given one, and what is asked of it
    auto of_bin = [&](Question q, uint32_t which, uint64_t t, double d, bool pick) {
        const bool given = q == kValue;
        if (given ? which / kOwn == threadIdx.x : before < t && t <= before + own) {
            uint64_t upto = before;
            for (uint32_t i = threadIdx.x * kOwn;; ++i) {
                const uint64_t here = s.mass[i];
                if (given ? i == which : t <= upto + here) {
                    s.bin = i;
                    s.before = upto;
                    break;
                }
                upto += here;
            }
        }
        __syncthreads();
        const uint32_t bin = s.bin;
        const uint64_t ahead = s.before;
        __syncthreads();
        const float lo = bins.lowest(bin);
        return through(r, q, lo > r.least ? lo : r.least, bins.highest(bin), ahead, t, d, pick);
    };
    if (a.by_mass) sum = of_bin(kMass, 0, a.share(sum), 0.0, false);
    if (a.by_value) {
        const float at = (float)(r.masses.max + a.border);
        if (at >= r.least) {
            const uint64_t kept = of_bin(kValue, bins(at), 0, a.border, false);
            sum = kept < sum ? kept : sum;
        }
    }
    (void)of_bin(kMass, 0, __umul64hi(a.u, sum) + 1, 0.0, true);
    __syncthreads();
    return sum;
}

// Rows in whose bins every logit is the same number: what is left is arithmetic, and the token the nth of a number.  Returns 0 if the answer hangs on what lies
// around 0, which may be several.
template <typename T, int THREADS, int N>
__device__ __forceinline__ uint64_t answer_by_numbers(const Row<T, THREADS>& r, const Kept<T, THREADS, N>& kept, const Asked& a, uint32_t k_bin, uint32_t k_left) {
    constexpr uint32_t E = Pieces<T>::E;
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    const Bins bins = fixed_bins();
    uint64_t zeros = 0;
    if (s.count[kFixedTop]) {
        const float tiny = bins.highest(kFixedTop);
        uint64_t mine = 0;
        bool some = false;
        r.stream([&](const float(&v)[E], uint32_t) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (fabsf(v[e]) <= tiny) {
                    mine += r.masses(v[e]);
                    some |= v[e] != 0.f;
                }
        });
        if (some) s.ahead = 1;
        (void)before_thread<THREADS>(mine, s.sums, zeros);
    }
    auto number = [&](uint32_t bin) { return bin == (uint32_t)kFixedTop ? 0.f : bins.number(bin); };
    auto mass = [&](uint32_t bin, uint32_t n) { return bin == (uint32_t)kFixedTop ? zeros : n * r.masses(bins.number(bin)); };
    r.sum_groups(mass);
    if (threadIdx.x < 64) {
        uint64_t sum = r.sum_before_groups();
        bool known = true;
        auto each_of = [&](uint32_t bin) {
            const uint64_t each = r.masses(number(bin));
            if (bin == (uint32_t)kFixedTop && s.ahead) known = false;
            return each;
        };
        if (a.k) {
            const auto f = r.find_bin(true, k_bin, 0, mass);
            sum = f.before + k_left * each_of(k_bin);
        }
        if (a.by_mass) {
            const uint64_t t = a.share(sum);
            const auto f = r.find_bin(false, 0, t, mass);
            const uint64_t each = each_of(f.bin);
            if (known) sum = f.before + (t - f.before + each - 1) / each * each;
        }
        if (a.by_value && known) {
            const float at = (float)(r.masses.max + a.border);
            if (at >= r.least && at > -kFixedMost) {
                const uint32_t bin = bins(at);
                const auto f = r.find_bin(true, bin, 0, mass);
                if (bin == (uint32_t)kFixedTop && f.here) (void)each_of(bin);
                const uint64_t to = f.before + ((double)number(bin) - r.masses.max >= a.border ? f.here : 0);
                sum = to < sum ? to : sum;
            }
        }
        if (known) {
            const uint64_t t = __umul64hi(a.u, sum) + 1;
            const auto f = r.find_bin(false, 0, t, mass);
            const uint64_t each = each_of(f.bin);
            if (known && threadIdx.x == 0) {
                s.value = number(f.bin);
                s.before = (t - f.before + each - 1) / each;
                s.ahead = s.count[f.bin];
            }
        }
        if (threadIdx.x == 0) s.through = known ? sum : 0;
    }
    __syncthreads();
    const uint64_t sum = s.through;
    if (sum) kept.find(s.value, s.before, s.ahead);
    return sum;
}

// The bin in which mass reaches t; s.mass holds what lies before each.
template <typename T, int THREADS>
__device__ __forceinline__ uint32_t bin_at_mass(uint64_t t) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    const uint32_t lane = threadIdx.x & 63, thirty = (uint32_t)__popcll(__ballot(s.mass[lane * 32] < t)) - 1;
    return uniform(thirty * 32 + (uint32_t)__popcll(__ballot(lane < 32 && s.mass[thirty * 32 + (lane & 31)] < t)) - 1);
}
// What lies before each bin takes the masses' place; returns the sum of all.
template <typename T, int THREADS>
__device__ __forceinline__ uint64_t sum_before_bins() {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    static_assert(kBins == 64 * 32);
    constexpr uint32_t kOwn = kBins / THREADS;
    uint64_t own[kOwn], mine = 0, all;
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i) {
        own[i] = s.mass[threadIdx.x * kOwn + i];
        mine += own[i];
    }
    uint64_t before = before_thread<THREADS>(mine, s.sums, all);
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i) {
        s.mass[threadIdx.x * kOwn + i] = before;
        before += own[i];
    }
    __syncthreads();
    return all;
}

// The bins that tell what is kept and which the token is, as far as bins tell, without top_k: s.mass holds what lies before each, `all` in all.
struct Wanted {
    uint32_t from, to, p_from, p_to, value;                       // of the token, of top_p (from > to: none) and of min_p (~0: none)
    uint64_t value_before;
    __device__ __forceinline__ bool operator()(uint32_t bin) const { return (bin >= from && bin <= to) || (bin >= p_from && bin <= p_to) || bin == value; }
};
template <typename T, int THREADS, typename B>
__device__ __forceinline__ Wanted wanted_bins(const Asked& q, uint64_t all, double max, float least, B bin_of) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    auto end_of = [&](uint32_t bin) { return bin + 1 < kBins ? s.mass[bin + 1] : all; };
    auto some = [](uint64_t v) { return v ? v : (uint64_t)1; };
    uint64_t fewest = all, most = all;                            // what is kept lies between these two
    Wanted w{0, 0, 1, 0, ~0u, 0};
    if (q.by_mass) {
        w.p_from = bin_at_mass<T, THREADS>(q.share(fewest));
        w.p_to = bin_at_mass<T, THREADS>(q.share(most));
        fewest = some(s.mass[w.p_from]);
        most = end_of(w.p_to);
    }
    if (q.by_value) {
        const float at = (float)(max + q.border);
        if (at >= least) {
            w.value = bin_of(at);
            w.value_before = s.mass[w.value];
            const uint64_t before = some(w.value_before), end = end_of(w.value);
            fewest = before < fewest ? before : fewest;
            most = end < most ? end : most;
        }
    }
    w.from = bin_at_mass<T, THREADS>(__umul64hi(q.u, fewest) + 1);
    w.to = bin_at_mass<T, THREADS>(__umul64hi(q.u, most) + 1);
    return w;
}
// Writes the answer out of a list of the n <= kList logits in the wanted bins: put in order by the workgroup, the rest by its first wave.
template <typename T, int THREADS, typename B>
__device__ __forceinline__ void finish_from_bins(const SampleShape& shape, uint64_t row, const Row<T, THREADS>& r, const Asked& a, const Wanted& wanted, uint64_t all, uint32_t n, B bin_of) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    sort_list<T, THREADS>(n);
    if (threadIdx.x >= 64) return;
    const uint32_t each = (n + 63) / 64, first = threadIdx.x * each;                       // in their order: `each` of a lane
    auto value = [&](uint32_t i) { return of_key((uint32_t)(s.sorted[i] >> 32)); };
    uint64_t sum = 0;
    for (uint32_t i = first; i < first + each && i < n; ++i) {
        sum += r.masses(value(i));
        s.upto[i] = sum;
    }
    const uint64_t before = upto_lane(sum) - sum;
    for (uint32_t i = first; i < first + each && i < n; ++i) s.upto[i] += before;
    wave_sync();
    // the list's sums leave out what lies between its bins: a bin's first logit puts that right, in the place of what lies before the bin
    for (uint32_t i = first; i < first + each && i < n; ++i)
        if (i == 0 || bin_of(value(i)) != bin_of(value(i - 1))) s.mass[bin_of(value(i))] -= i ? s.upto[i - 1] : 0;
    wave_sync();
    for (uint32_t i = first; i < first + each && i < n; ++i) s.upto[i] += s.mass[bin_of(value(i))];
    wave_sync();
    auto places = [&](auto f) {                                   // at which f is true, which are the first ones
        uint32_t count = 0;
        for (uint32_t i = 0; i < n; i += 64) count += (uint32_t)__popcll(__ballot(i + threadIdx.x < n && f(i + threadIdx.x)));
        return count;
    };
    auto reached = [&](uint64_t t) { return places([&](uint32_t i) { return s.upto[i] < t; }); };
    sum = all;
    if (a.by_mass) sum = s.upto[reached(a.share(sum))];
    if (wanted.value != ~0u) {
        const uint32_t kept = places([&](uint32_t i) { return (double)value(i) - r.masses.max >= a.border; });
        const uint64_t to = kept && bin_of(value(kept - 1)) == wanted.value ? s.upto[kept - 1] : wanted.value_before;
        sum = to < sum ? to : sum;
    }
    const uint64_t token = s.sorted[reached(__umul64hi(a.u, sum) + 1)];
    if (threadIdx.x == 0) write_answer(shape, row, a, r.masses, ~(uint32_t)token, of_key((uint32_t)(token >> 32)), sum);
}

// Rows of any numbers between the fixed bins' ends, without top_k: masses of four bins at a time.  Returns false if the list is too short.
template <typename T, int THREADS, int N>
__device__ __forceinline__ bool finish_by_masses(const SampleShape& shape, uint64_t row, const Row<T, THREADS>& r, const Kept<T, THREADS, N>& kept, const Asked& a) {
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    static_assert(kBins * 4 == kFixedBins);
    const Bins bins = fixed_bins();
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kBins; i += THREADS) s.mass[i] = 0;
    __syncthreads();
    kept.of_all([&](float v) {
        if (v >= r.least) atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[(bins(v) - kFixedFirst) / 4]), (unsigned long long)r.masses(v));
    });
    __syncthreads();
    const uint64_t all = sum_before_bins<T, THREADS>();
    auto bin_of = [&](float v) { return (bins(v) - kFixedFirst) / 4; };
    const Wanted wanted = wanted_bins<T, THREADS>(a, all, r.masses.max, r.least, bin_of);
    // as limits of logits: the token's bins, and those of top_p and of min_p
    auto low = [&](uint32_t g) { return fmaxf(bins.lowest(kFixedFirst + 4 * g + 3), r.least); };
    auto high = [&](uint32_t g) { return bins.highest(kFixedFirst + 4 * g); };
    const float lo0 = low(wanted.to), hi0 = high(wanted.from), none = kInf;
    const float lo1 = a.by_mass ? low(wanted.p_to) : none, hi1 = a.by_mass ? high(wanted.p_from) : -none;
    const float lo2 = wanted.value != ~0u ? low(wanted.value) : none, hi2 = wanted.value != ~0u ? high(wanted.value) : -none;
    const uint32_t n = kept.gather_those([&](float v) { return (v >= lo0 && v <= hi0) || (v >= lo1 && v <= hi1) || (v >= lo2 && v <= hi2); });
    if (n > kList) return false;
    finish_from_bins(shape, row, r, a, wanted, all, n, bin_of);
    return true;
}

template <typename T, int THREADS, int N, int WAVES>
__global__ void __launch_bounds__(THREADS, WAVES) sample_kernel(SampleShape a) {
    constexpr bool kNumbers = Row<T, THREADS>::kNumbers;
    SampleLds<THREADS>& s = sample_lds<T, THREADS>();
    const uint64_t row = a.row0 + blockIdx.x;
    Row<T, THREADS> r{static_cast<const T*>(a.z) + row * a.z_ld, (uint32_t)a.vocab, {}, 0.f};
    const Kept<T, THREADS, N> kept(r.z, r.vocab);
    Asked asked = asked_of(a, row);
    if (threadIdx.x == 0) s.index = 0;
    // the largest, and how many logits are in each of the fixed bins
    const bool counted = kNumbers || asked.k;
    float max = -kInf;
    bool known = !counted || !kNumbers;                           // max is the largest, or will be
    uint32_t first = 0;                                           // counted: the bin of the largest
    const float u_given = a.u[row], min_p = a.each.min_p_dev ? a.each.min_p_dev[row] : a.min_p;       // (asked for with the row)
    if (counted) {
        u32x4* const clear = reinterpret_cast<u32x4*>(s.count);
        for (uint32_t i = threadIdx.x; i < kFixedCounts / 4; i += THREADS) clear[i] = u32x4{0, 0, 0, 0};
        r.clear_groups();
        if (threadIdx.x == 0) s.held = s.ahead = 0;               // (ahead: there are numbers around 0 that are not 0)
        __syncthreads();
        const auto c = kept.count_fixed();
        max = c.max;
        if constexpr (kNumbers) {
            // no number is beyond the bins (NaN is), and the first that is not empty tells the largest, unless it is the one around 0
            if (c.nan) s.held = 1;
            __syncthreads();
            first = r.first_bin();
            known = first > kFixedFirst && first < kFixedLast && first != (uint32_t)kFixedTop && uniform(s.held) == 0;
            if (known) max = fixed_bins().number(first);
        }
    }
    if (!counted || (kNumbers && !known)) max = kept.largest();
    if (!kNumbers || !counted || !known) {
        max = over_lanes<64>(max, [](float x, float y) { return max_or_nan(x, y); });
        if ((threadIdx.x & 63) == 0) s.most[threadIdx.x / 64] = max;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) max = max_or_nan(max, s.most[w]);
    }
    max = uniform(max);
    if (max != max || max == -kInf) {
        if (threadIdx.x == 0) no_answer(a, row, max);
        return;
    }
    ask(a, max, u_given, min_p, asked, r.masses, r.least);
    const bool fixed = counted && max < kFixedMost && r.least > -kFixedMost;
    bool listed = false;                                          // everything that matters lies above r.least, and the list has room for it
    if (asked.by_value && !asked.by_mass) {                       // no other filter needs what this one leaves out
        const float at = (float)((double)max + asked.border), below = at - (fabsf(at) + fabsf(max)) * 0x1p-20f;
        if (below > r.least) r.least = below;
    }
    float k_low = 0.f, k_high = 0.f;
    uint32_t k_bin = 0, k_left = 0;
    if (fixed && asked.k) {
        // from the largest one's bin on, 64 bins at a time, every wave by itself; where that is long, by groups
        uint32_t ahead = 0, here = 0;
        bool there = false;
        k_bin = kNumbers && known ? first : uniform(fixed_bins()(max));
        for (int step = 0; step < 12 && !there && k_bin < kFixedLast; ++step) {
            const uint32_t n = r.fixed_count(k_bin + (threadIdx.x & 63)), upto = upto_lane(n), all = (uint32_t)__builtin_amdgcn_readlane(upto, 63);
            if (ahead + all >= asked.k) {
                const uint32_t at = (uint32_t)__builtin_ctzll(__ballot(ahead + upto >= asked.k));
                here = (uint32_t)__builtin_amdgcn_readlane(n, at);
                ahead += (uint32_t)__builtin_amdgcn_readlane(upto, at) - here;
                k_bin += at;
                there = true;
            } else {
                ahead += all;
                k_bin += 64;
            }
        }
        if (!there && k_bin >= kFixedLast) {                      // there are no more than k
            asked.k = 0;
        } else if (!there) {
            auto count = [](uint32_t, uint32_t n) { return (uint64_t)n; };
            r.sum_groups(count);
            if (threadIdx.x < 64) {
                const uint64_t all = r.sum_before_groups();
                uint32_t bin = ~0u;
                if (asked.k < all) {
                    const auto f = r.find_bin(false, 0, asked.k, count);
                    bin = f.bin;
                    ahead = (uint32_t)f.before;
                    here = (uint32_t)f.here;
                }
                if (threadIdx.x == 0) {
                    s.bin = bin;
                    s.least = ahead;
                    s.held = here;
                }
            }
            __syncthreads();
            k_bin = uniform(s.bin);
            ahead = uniform(s.least);
            here = uniform(s.held);
            if (k_bin == ~0u) asked.k = 0;
            r.clear_groups();
            __syncthreads();
        }
        if (asked.k) {
            k_left = asked.k - ahead;
            listed = ahead + here <= kList;
            k_low = fixed_bins().lowest(k_bin);
            k_high = fixed_bins().highest(k_bin);
            if (listed && k_low > r.least) r.least = k_low;
        }
    }
    if (listed || (!kNumbers && asked.by_value && !asked.by_mass && !asked.k)) {
        const uint32_t n = kept.gather(r.least, kInf);
        if (n <= kList) return finish_from_list(a, row, r, asked, n);
    }
    uint64_t sum = 0;
    if constexpr (kNumbers)
        if (fixed) sum = answer_by_numbers(r, kept, asked, k_bin, k_left);
    if constexpr (!kNumbers && (N <= 8 || (N <= 16 && WAVES <= 3)))                        // (others have no registers left)
        if (max < kFixedMost && r.least > -kFixedMost && !asked.k)
            if (finish_by_masses(a, row, r, kept, asked)) return;
    if (!sum) sum = answer_any(r, asked.temperature, asked.top_p, max, asked.k, asked.u, asked.border, k_low, k_high, k_left);
    if (threadIdx.x == 0) write_answer(a, row, asked, r.masses, s.index, (float)r.z[s.index], sum);
}

// Short rows: a wave each, with the row in LDS.  Bins are linear between what is looked for and divided again as long as more than 64 logits that are not alike lie in
// the one that matters.
constexpr uint32_t kWaveRows = 4;
template <uint32_t ROOM>
struct WaveLds {
    uint64_t mass[kWaveBins], list[64];
    uint32_t count[kWaveBins];
    float z[ROOM];
};
template <typename T, uint32_t ROOM>
__global__ void __launch_bounds__(64 * kWaveRows) sample_wave_kernel(SampleShape a, uint64_t rows_end) {
    constexpr uint32_t E = Pieces<T>::E, kOwn = kWaveBins / 64, kStep = 4 * 64;
    using Piece = typename Pieces<T>::Piece;
    __shared__ WaveLds<ROOM> lds[kWaveRows];
    WaveLds<ROOM>& s = lds[threadIdx.x / 64];
    const uint32_t lane = threadIdx.x & 63, vocab = (uint32_t)a.vocab;
    const uint64_t row = a.row0 + (uint64_t)blockIdx.x * kWaveRows + uniform(threadIdx.x / 64);
    if (row >= rows_end) return;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    const uint32_t end = (vocab + kStep - 1) / kStep * kStep;    // filled with minus infinity
    float max = -kInf;
    for (uint32_t at = lane * E; at < end; at += 64 * E) {
        float v[E];
        if (at + E <= vocab) {
            const Piece piece = *reinterpret_cast<const Piece*>(z + at);
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) v[e] = (float)piece[e];
        } else {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) v[e] = at + e < vocab ? (float)z[at + e] : -kInf;
        }
        max = max_or_nan(max, largest_of(v));
#pragma unroll
        for (uint32_t e = 0; e < E; e += 4) *reinterpret_cast<f32x4*>(s.z + at + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    }
    Asked q = asked_of(a, row);
    const float u = a.u[row], min_p = a.each.min_p_dev ? a.each.min_p_dev[row] : a.min_p;
    // f(logit, column), kept together four times 64 at once; the first ones first
    auto of_all = [&](auto f) {
#pragma unroll 1
        for (uint32_t at = lane; at < end; at += kStep) {
            float x[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) x[i] = s.z[at + i * 64];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) f(x[i], at + i * 64);
        }
    };
    auto smaller = [](float x, float y) { return x < y ? x : y; };
    auto larger = [](float x, float y) { return x > y ? x : y; };
    auto plus = [](uint32_t x, uint32_t y) { return x + y; };
    max = uniform(over_lanes<64>(max, [](float x, float y) { return max_or_nan(x, y); }));
    wave_sync();
    if (max != max || max == -kInf) {
        if (lane == 0) no_answer(a, row, max);
        return;
    }
    Masses masses;
    float least;
    ask(a, max, u, min_p, q, masses, least);
    if (q.infinite) {                                             // as zeros among minus infinities
        for (uint32_t at = lane; at < end; at += 64) s.z[at] = s.z[at] == kInf ? 0.f : -kInf;
        masses.max = 0.0;
        masses.least = -1000.0;
        least = 0.f;
        wave_sync();
    }
    LinearBins bin_of{masses.max, 0.0, 0.0};
    auto distance = [&](float x) { return bin_of.distance(x); };

    // bins of the logits from lo to hi, at level 0 from the lowest that has mass to the largest
    float lo = kInf, hi = q.infinite ? 0.f : max;
    uint32_t n = 0;
    of_all([&](float x, uint32_t) {
        if (x >= least) {
            lo = smaller(lo, x);
            ++n;
        }
    });
    lo = uniform(over_lanes<64>(lo, smaller));
    n = uniform(over_lanes<64>(n, plus));
    if (q.k >= n) q.k = 0;
    uint64_t own[kOwn], before;                                   // masses of the lane's bins, and before them
    uint32_t own_count[kOwn], count_before;
    auto fill_bins = [&] {
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) {
            s.mass[i * 64 + lane] = 0;
            s.count[i * 64 + lane] = 0;
        }
        wave_sync();
        of_all([&](float x, uint32_t) {
            if (x >= lo && x <= hi) {
                const uint32_t bin = bin_of(x);
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[bin]), (unsigned long long)masses(x));
                atomicAdd(&s.count[bin], 1u);
            }
        });
        wave_sync();
        uint64_t sum = 0;
        uint32_t count = 0;
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) {
            own[i] = s.mass[lane * kOwn + i];
            own_count[i] = s.count[lane * kOwn + i];
            sum += own[i];
            count += own_count[i];
        }
        before = upto_lane(sum) - sum;
        count_before = upto_lane(count) - count;
        wave_sync();
    };
    const float lowest = lo, highest = hi;
    uint32_t index = 0;
    float value = 0.f;
    uint64_t sum = 0;
    bool whole = false;                                           // the bins are those of level 0
    for (int step = 0; step < 4; ++step) {                        // top_k, or the sum of all that others start from; top_p, min_p, the token
        if ((step == 1 && !q.by_mass) || (step == 2 && !q.by_value)) continue;
        lo = lowest;
        hi = highest;
        uint64_t ahead = 0, t = step == 0 ? q.k : step == 1 ? q.share(sum) : __umul64hi(q.u, sum) + 1;
        uint32_t here = n;                                        // logits from lo to hi
        bool first = true, one = lo == hi;                        // one: logits from lo to hi are alike (at first, when hi is the largest: equal)
        uint64_t through = 0;
        for (;;) {
            if (__builtin_expect(one, 0)) {                       // all of the same mass
                const uint64_t each = masses(lo);
                const uint64_t nth = step == 0 ? (q.k ? t : here) : step == 2 ? (-distance(lo) >= q.border ? here : 0) : (t - ahead + each - 1) / each;
                through = ahead + nth * each;
                if (step == 3) {
                    uint32_t left = (uint32_t)nth;
                    if (lo != hi) {                               // which number it is, and the how-manieth of these
                        auto above = [&](uint32_t key) {          // logits from this key to hi
                            uint32_t count = 0;
                            of_all([&](float x, uint32_t) { count += x <= hi && logit_key(x) >= key ? 1u : 0u; });
                            return uniform(over_lanes<64>(count, plus));
                        };
                        NthKey keys{logit_key(lo), logit_key(hi)};
                        while (!keys.done()) keys.counted(above(keys.tried()) >= left);
                        left -= above(keys.low + 1);
                        lo = of_key(keys.low);
                    }
                    value = lo;
                    of_all([&](float x, uint32_t column) {
                        const uint64_t those = __ballot(x == lo);
                        const uint32_t all = (uint32_t)__popcll(those);
                        if (left && left <= all) {
                            const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(those >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)those, 0));
                            index = (uint32_t)__builtin_amdgcn_readlane(column, __builtin_ctzll(__ballot(x == lo && below == left - 1)));
                        }
                        left = left <= all ? 0 : left - all;
                    });
                }
                break;
            }
            if (here <= 64) {                                     // one of them a lane, in their order
                uint32_t held = 0;
                of_all([&](float x, uint32_t column) {
                    const bool in = x >= lo && x <= hi;
                    const uint64_t those = __ballot(in);
                    if (in) s.list[held + __builtin_amdgcn_mbcnt_hi((uint32_t)(those >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)those, 0))] = logit_rank(x, column);
                    held += (uint32_t)__popcll(those);
                });
                wave_sync();
                const uint64_t mine = lane < here ? s.list[lane] : 0;
                uint32_t place = 0;
                for (uint32_t j = 0; j < here; ++j) place += s.list[j] > mine ? 1u : 0u;
                wave_sync();
                if (lane < here) s.list[place] = mine;
                wave_sync();
                const uint64_t rank = lane < here ? s.list[lane] : 0;
                const float x = of_key((uint32_t)(rank >> 32));
                const uint64_t upto = ahead + upto_lane(lane < here ? masses(x) : 0);
                wave_sync();
                uint32_t at;                                      // of the last that is kept, or of the token; here: none
                if (step == 0) at = (q.k ? (uint32_t)t : here) - 1;
                else if (step == 2) at = (uint32_t)__popcll(__ballot(lane < here && -distance(x) >= q.border)) - 1;
                else at = (uint32_t)__builtin_ctzll(__ballot(lane < here && upto >= t));
                through = at == ~0u ? ahead : of_lane(upto, at);
                if (step == 3) {
                    index = ~(uint32_t)__builtin_amdgcn_readlane((uint32_t)rank, at);
                    value = uniform(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at)));
                }
                break;
            }
            if (!(first && whole)) {
                bin_of.set(lo, hi);
                bin_of.scale = uniform(bin_of.scale);
                fill_bins();
                whole = first;
            }
            if (step == 0 && !q.k) {                              // all of it
                uint64_t mine = 0;
#pragma unroll
                for (uint32_t i = 0; i < kOwn; ++i) mine += own[i];
                through = of_lane(before + mine, 63);
                break;
            }
            // the bin
            uint32_t which = 0, inside = 0;
            uint64_t upto = ahead + before;
            bool it = false;
            if (step == 2) {
                const double d = -q.border;
                const double place = (d - bin_of.from) * bin_of.scale;
                const uint32_t bin = place <= 0.0 ? 0 : place >= kWaveBins ? kWaveBins - 1 : (uint32_t)place;
#pragma unroll
                for (uint32_t i = 0; i < kOwn; ++i) {
                    if (lane * kOwn + i == bin) {
                        it = true;
                        which = i;
                        inside = own_count[i];
                    }
                    if (!it) upto += own[i];
                }
            } else {
                uint32_t counted = count_before;
#pragma unroll
                for (uint32_t i = 0; i < kOwn; ++i) {
                    const bool reached = step == 0 ? counted < t && t <= counted + own_count[i] : upto < t && t <= upto + own[i];
                    if (reached && !it) {
                        it = true;
                        which = i;
                        inside = own_count[i];
                    }
                    if (!it) {
                        upto += own[i];
                        counted += own_count[i];
                    }
                }
                if (step == 0 && it) t -= counted;
            }
            const uint32_t owner = (uint32_t)__builtin_ctzll(__ballot(it));
            const uint32_t bin = owner * kOwn + (uint32_t)__builtin_amdgcn_readlane(which, owner);
            here = (uint32_t)__builtin_amdgcn_readlane(inside, owner);
            ahead = of_lane(upto, owner);
            if (step == 0) t = of_lane(t, owner);
            if (here == 0) {
                through = ahead;
                break;
            }
            float low = kInf, high = -kInf;
            of_all([&](float x, uint32_t) {
                if (x >= lo && x <= hi && bin_of(x) == bin) {
                    low = smaller(low, x);
                    high = larger(high, x);
                }
            });
            lo = uniform(over_lanes<64>(low, smaller));
            hi = uniform(over_lanes<64>(high, larger));
            first = false;
            one = bin_of.alike(lo, hi);
        }
        if (step == 2) sum = through < sum ? through : sum;
        else if (step < 2) sum = through;
    }
    if (lane == 0) write_answer(a, row, q, masses, index, value, sum);
}

// Few long rows are split over workgroups, in four launches: the largest of each part; masses in bins of the row, added up in memory; which bins matter, as far as they tell, and the
// logits in them into a list of the row; the answer out of bins and list.  A row with a top_k after all (of its own), or with a list too long, is the last launch's alone.
constexpr uint32_t kSplitThreads = 256;
struct SplitRow {
    uint64_t mass[kBins];
    uint64_t list[kList];
    float most[64];                                               // of parts
    uint32_t held, unused[3];
};
struct SplitShape : SampleShape {
    SplitRow* rows_of;
    uint32_t parts, part_logits;                                  // parts <= 64; part_logits: a multiple of what 16 bytes hold
};
template <typename T>
__device__ __forceinline__ Row<T, kSplitThreads> part_of(const SplitShape& a) {
    const uint32_t begin = blockIdx.x * a.part_logits, vocab = (uint32_t)a.vocab;
    Row<T, kSplitThreads> r{};
    r.z = static_cast<const T*>(a.z) + (a.row0 + blockIdx.y) * a.z_ld + begin;
    r.vocab = vocab - begin < a.part_logits ? vocab - begin : a.part_logits;
    return r;
}
__device__ __forceinline__ float split_largest(const SplitShape& a, const SplitRow& w) {
    const uint32_t lane = threadIdx.x & 63;
    return uniform(over_lanes<64>(lane < a.parts ? w.most[lane] : -kInf, [](float x, float y) { return max_or_nan(x, y); }));
}
template <typename T>
__device__ __forceinline__ void split_ask(const SplitShape& a, float max, Asked& q, Masses& masses, float& least) {
    const uint64_t row = a.row0 + blockIdx.y;
    q = asked_of(a, row);
    ask(a, max, a.u[row], a.each.min_p_dev ? a.each.min_p_dev[row] : a.min_p, q, masses, least);
}

// What lies in memory since the launch before is asked for at once, before anything is made of it: a read takes a microsecond.
struct SplitMasses {
    static constexpr uint32_t kEach = kBins / kSplitThreads;
    uint64_t mass[kEach];
    __device__ __forceinline__ explicit SplitMasses(const SplitRow& w) {
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) mass[i] = w.mass[i * kSplitThreads + threadIdx.x];
    }
    __device__ __forceinline__ void put(uint64_t* to) const {
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) to[i * kSplitThreads + threadIdx.x] = mass[i];
        __syncthreads();
    }
};

template <typename T>
__global__ void __launch_bounds__(kSplitThreads) sample_most_kernel(SplitShape a) {
    constexpr uint32_t E = Pieces<T>::E;
    __shared__ float most[kSplitThreads / 64];
    SplitRow& w = a.rows_of[blockIdx.y];
    const auto r = part_of<T>(a);
    for (uint32_t i = blockIdx.x * kSplitThreads + threadIdx.x; i < kBins; i += gridDim.x * kSplitThreads) w.mass[i] = 0;
    float max = -kInf;
    r.stream([&](const float(&v)[E], uint32_t) { max = max_or_nan(max, largest_of(v)); });
    max = over_lanes<64>(max, [](float x, float y) { return max_or_nan(x, y); });
    if ((threadIdx.x & 63) == 0) most[threadIdx.x / 64] = max;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (uint32_t i = 1; i < kSplitThreads / 64; ++i) max = max_or_nan(max, most[i]);
    w.most[blockIdx.x] = max;
    if (blockIdx.x == 0) w.held = 0;
}

template <typename T>
__global__ void __launch_bounds__(kSplitThreads) sample_bins_kernel(SplitShape a) {
    constexpr uint32_t E = Pieces<T>::E;
    __shared__ uint64_t mass[kBins];
    SplitRow& w = a.rows_of[blockIdx.y];
    for (uint32_t i = threadIdx.x; i < kBins; i += kSplitThreads) mass[i] = 0;
    const float max = split_largest(a, w);
    if (max != max || max == -kInf) return;
    auto r = part_of<T>(a);
    Asked q;
    split_ask<T>(a, max, q, r.masses, r.least);
    const Bins bins = bins_of(max, q.temperature);
    __syncthreads();
    r.stream([&](const float(&v)[E], uint32_t) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
            if (v[e] >= r.least) atomicAdd(reinterpret_cast<unsigned long long*>(&mass[bins(v[e])]), (unsigned long long)r.masses(v[e]));
    });
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kBins; i += kSplitThreads)
        if (mass[i]) atomicAdd(reinterpret_cast<unsigned long long*>(&w.mass[i]), (unsigned long long)mass[i]);
}

template <typename T>
__global__ void __launch_bounds__(kSplitThreads) sample_sift_kernel(SplitShape a) {
    constexpr uint32_t E = Pieces<T>::E;
    SampleLds<kSplitThreads>& s = sample_lds<T, kSplitThreads>();
    SplitRow& w = a.rows_of[blockIdx.y];
    const SplitMasses masses(w);
    const float max = split_largest(a, w);
    if (max != max || max == -kInf) return;
    auto r = part_of<T>(a);
    Asked q;
    split_ask<T>(a, max, q, r.masses, r.least);
    const Bins bins = bins_of(max, q.temperature);
    masses.put(s.mass);
    const uint64_t all = sum_before_bins<T, kSplitThreads>();
    const Wanted wanted = wanted_bins<T, kSplitThreads>(q, all, r.masses.max, r.least, bins);
    // the part's into LDS, where masses are done with, and then with one request for places into the row's
    __syncthreads();
    if (threadIdx.x == 0) s.held = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * a.part_logits;
    r.stream([&](const float(&v)[E], uint32_t at) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
            if (v[e] >= r.least) {
                if (wanted(bins(v[e]))) {
                    const uint32_t place = atomicAdd(&s.held, 1u);
                    if (place < kBins) s.mass[place] = logit_rank(v[e], begin + at + e);
                }
            }
    });
    __syncthreads();
    const uint32_t held = s.held;
    if (held == 0) return;
    if (threadIdx.x == 0) s.ahead = atomicAdd(&w.held, held);
    __syncthreads();
    const uint32_t first = s.ahead;
    for (uint32_t i = threadIdx.x; i < held && i < kBins && first + i < kList; i += kSplitThreads) w.list[first + i] = s.mass[i];
}

template <typename T>
__global__ void __launch_bounds__(kSplitThreads, 4) sample_split_kernel(SplitShape a) {
    SampleLds<kSplitThreads>& s = sample_lds<T, kSplitThreads>();
    SplitRow& w = a.rows_of[blockIdx.y];
    const uint64_t row = a.row0 + blockIdx.y;
    const SplitMasses masses(w);
    constexpr uint32_t kEach = kList / kSplitThreads;
    uint64_t rank[kEach];                                         // the thread's part of the list
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) rank[i] = w.list[i * kSplitThreads + threadIdx.x];
    const uint32_t listed = w.held;
    const float max = split_largest(a, w);
    if (max != max || max == -kInf) {
        if (threadIdx.x == 0) no_answer(a, row, max);
        return;
    }
    Row<T, kSplitThreads> r{static_cast<const T*>(a.z) + row * a.z_ld, (uint32_t)a.vocab, {}, 0.f};
    Asked q;
    split_ask<T>(a, max, q, r.masses, r.least);
    if (q.k || listed > kList) {
        if (threadIdx.x == 0) s.index = 0;
        const uint64_t sum = answer_any(r, q.temperature, q.top_p, max, q.k, q.u, q.border, 0.f, 0.f, 0u);
        if (threadIdx.x == 0) write_answer(a, row, q, r.masses, s.index, (float)r.z[s.index], sum);
        return;
    }
    const Bins bins = bins_of(max, q.temperature);
    masses.put(s.mass);
    const uint64_t all = sum_before_bins<T, kSplitThreads>();
    const Wanted wanted = wanted_bins<T, kSplitThreads>(q, all, r.masses.max, r.least, bins);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
        if (i * kSplitThreads + threadIdx.x < listed) s.list[i * kSplitThreads + threadIdx.x] = rank[i];
    __syncthreads();
    finish_from_bins(a, row, r, q, wanted, all, listed, bins);
}

// Workgroups of a row, 1 for none.  Of bf16, and where top_k or min_p alone leave little, a workgroup by itself reads a row twice at most: 1 x 131072, bf16, top_p, 22 us,
// split 30; 4 x 131072, fp32, min_p, 14.5 and 24.6.  Otherwise it reads it four times and makes masses of all of it: 1 x 131072, fp32, top_p, 88 us, split 25; 32 x 40000 42 and 34; 4 x 20000 25 and 28.
// At temperature 0, where the largest is all that is kept, a workgroup as well: 1 x 131072, fp32, 18 and 61, 1 x 8 million 1008 and 3637.
uint32_t sample_parts(const ds_sampling& l) {
    const uint64_t size = l.dtype == DS_F32 ? 4 : 2, bytes = l.vocab * size;
    const bool few_left = l.dtype == DS_BF16 || (l.min_p > 0.f && l.top_p >= 1.f);
    if (l.top_k > 0 || l.temperature == 0.f || l.rows > 32 || bytes < (few_left ? 1u << 20 : 1u << 17)) return 1;
    const uint64_t p = (bytes + 16383) / 16384;
    return (uint32_t)(p < 64 ? p : 64);
}

template <int V>
using Int = std::integral_constant<int, V>;

template <typename T>
void launch_sample_of(const SampleArgs& args, hipStream_t stream) {
    SplitShape a{};
    static_cast<SampleArgs&>(a) = args;
    a.parts = a.work ? sample_parts({a.rows, a.vocab, a.dtype, a.top_k, a.temperature, a.top_p, a.min_p, 0}) : 1;
    if (a.parts > 1) {
        constexpr uint64_t E = Pieces<T>::E;
        a.rows_of = static_cast<SplitRow*>(a.work);
        a.part_logits = (uint32_t)(((a.vocab + a.parts - 1) / a.parts + E - 1) / E * E);
        a.parts = (uint32_t)((a.vocab + a.part_logits - 1) / a.part_logits);
        const dim3 grid(a.parts, (unsigned)a.rows), block(kSplitThreads);
        hipLaunchKernelGGL(sample_most_kernel<T>, grid, block, 0, stream, a);
        hipLaunchKernelGGL(sample_bins_kernel<T>, grid, block, 0, stream, a);
        hipLaunchKernelGGL(sample_sift_kernel<T>, grid, block, 0, stream, a);
        hipLaunchKernelGGL(sample_split_kernel<T>, dim3(1, (unsigned)a.rows), block, 0, stream, a);
        return;
    }
    for (uint64_t r = 0; r < a.rows; r += kRowsOfLaunch) {
        a.row0 = r;
        const unsigned here = (unsigned)(a.rows - r < kRowsOfLaunch ? a.rows - r : kRowsOfLaunch);
        auto launch = [&](auto threads, auto pieces, auto waves) {
            hipLaunchKernelGGL((sample_kernel<T, decltype(threads)::value, decltype(pieces)::value, decltype(waves)::value>), dim3(here), dim3(threads.value), 0, stream, a);
        };
        auto launch_waves = [&](auto room) {
            hipLaunchKernelGGL((sample_wave_kernel<T, decltype(room)::value>), dim3((here + kWaveRows - 1) / kWaveRows), dim3(64 * kWaveRows), 0, stream, a, r + here);
        };
        constexpr bool kWaves = !std::is_same_v<T, __bf16>;
        // A wave for a row: 64 x 500, fp32, top_p, 11.1 us (a workgroup 23), 4000 x 500 18.6 (111).  Above, for many rows of which masses have to be made: 4000 x 2000, fp32, top_p, 47.6
        // (53.8); but 1024 x 2000 24.7 (17.6), and 4000 x 2000, bf16, top_k, 54 (33).
        const uint64_t bytes = a.vocab * sizeof(T);
        const bool many = a.rows > 512, sums = kWaves && a.top_k == 0 && !(a.min_p > 0.f && a.top_p >= 1.f);
        if (a.vocab <= 512) launch_waves(Int<512>());
        else if (kWaves && a.vocab <= 2048 && a.rows >= 2048 && a.top_k == 0) launch_waves(Int<kWaves ? 2048 : 512>());
        else if (bytes <= 256 * 8 * 16) launch(Int<256>(), Int<8>(), Int<4>());
        // Of rows that a workgroup of 256 holds, three are on a compute unit instead of two, so that one counts while others go through the short phases behind that: 4096 x 16000, fp32,
        // k = 50, 68 us, so 59; 4096 x 32003, fp16, min_p, 71 and 51; 8000 x 32003, bf16, 227 and 193; but 1 x 32003, fp16, top_p, 36.6 and 38.0, 512 x 20000, bf16, 17.8 and 19.3.  Where masses of all
        // logits are made there is room for it in line, too (`answer_any` otherwise): 4096 x 16000, fp32, p = 0.9, 329 and 162; 4096 x 32003 462 and 322; but 4096 x 60000, fp16, 604 and 638.
        else if (many && (bytes <= 256 * 16 * 16 || (sums && a.vocab <= 32768))) launch(Int<256>(), Int<16>(), Int<3>());
        // Longer ones: 4096 x 24000, fp32, k = 50, 83 and 69; 2048 x 50001, bf16, 78.3 and 75.6; 4096 x 131072 252 and 246, 6144 rows 358 and 345, 8192 469 and 457; but 4096 x 28000, fp32, min_p, 78 and 84;
        // 1024 x 131072, bf16, 82 and 87, 2048 137 and 142, 3500 215 and 217.
        else if (bytes <= 256 * 24 * 16 ? a.rows > 1024 : !kWaves && a.rows >= (bytes <= 1u << 17 ? 2048u : 4096u)) launch(Int<256>(), Int<24>(), Int<3>());
        else launch(Int<512>(), Int<16>(), Int<4>());
    }
}

}  // namespace

uint64_t sample_work_bytes(const ds_sampling& s) {
    return sample_parts(s) > 1 ? s.rows * sizeof(SplitRow) : 0;
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_sample_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
