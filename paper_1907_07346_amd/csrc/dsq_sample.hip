// A token of every row of logits from a given random number (ds_sample).
//
// A row's order (larger first, of equal ones the lower index) is never made.  Every filter keeps a beginning of it, so that all that is needed of a filter is the
// mass of what it keeps, and the token is where the mass passes u times the smallest of these.  Each is one question: at which place of the order do count
// or mass reach a number?  Bins that follow the order answer it but for what lies in one bin, whose logits are then gathered, ranked and summed.
//   Masses exp((z - max) / T) are whole numbers of 2^-kBits or so, made in 64 bits: their sums are exact, so that they depend on no order, may be made with
// atomics, and differ from the formula's by less than 1e-13 of the largest one's mass per logit.  (A token is wrong where u comes closer to a border than the sums
// are off: with sums in 32 bits in one row of ten of 131072 logits.)
//   A workgroup takes a row, and reads it again for each stage: the largest; the bins; what lies in the bins that matter.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

constexpr uint64_t kRowsOfLaunch = 1u << 21;                      // a launch dimension holds fewer than 2^32 work-items
constexpr uint32_t kBins = 4096, kList = 512, kParts = 256;       // bins of a row; logits that are ranked at once; bins of a bin
constexpr uint32_t kAbove = 1536, kOctaves = 1024;                // bins for the logits of the largest one's sign; how far below T they are told apart
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

// Which bin of the row a logit lies in: bins are numbers of the 15 leading bits of its magnitude, those below `base` as one.
struct Bins {
    int32_t base, top;
    __device__ __forceinline__ uint32_t operator()(float z) const {
        const uint32_t bits = __float_as_uint(z);
        int32_t c = (int32_t)(bits >> 16 & 0x7FFFu) - base;
        c = c > 0 ? c : 0;
        const uint32_t bin = (uint32_t)(top - ((int32_t)bits < 0 ? -c : c));
        return bin < kBins - 1 ? bin : kBins - 1;
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
        if (bin == kBins - 1) return -kInf;
        if (v > 0) return __uint_as_float((uint32_t)(base + v) << 16);
        const uint32_t bits = (uint32_t)(base - v) << 16 | 0xFFFFu;
        return -__uint_as_float(bits < 0x7F800000u ? bits : 0x7F800000u);
    }
    // The only number of a bin, if logits have 8 bits ...
    __device__ __forceinline__ float number(uint32_t bin) const { return (int32_t)bin < top ? lowest(bin) : highest(bin); }
    // ... and this is true.
    __device__ __forceinline__ bool single(uint32_t bin) const { return bin != (uint32_t)top && bin != kBins - 1; }
};
__device__ __forceinline__ Bins bins_of(float max, float temperature) {
    const int32_t m = (int32_t)(__float_as_uint(max) >> 16 & 0x7FFFu), t = (int32_t)(__float_as_uint(temperature) >> 16) - (int32_t)kOctaves;
    Bins b;
    b.base = max < 0.f ? m : m - (int32_t)kAbove;
    if (b.base < t) b.base = t;
    if (b.base < 0) b.base = 0;
    if (b.base > 0x7F7F) b.base = 0x7F7F;
    const int32_t c = m > b.base ? m - b.base : 0;
    b.top = max < 0.f ? -c : c;
    return b;
}
__device__ __forceinline__ float of_key(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

template <int THREADS>
struct SampleLds {
    union {
        uint64_t mass[kBins];
        uint32_t count[2 * kBins];
    };
    uint64_t list[kList], sorted[kList], upto[kList];             // ranks of the logits gathered; in order; the mass through each
    uint64_t part_mass[kParts];
    uint32_t part_count[kParts];
    uint64_t sums[THREADS / 64];
    uint32_t counts[THREADS / 64];
    float most[THREADS / 64];
    uint64_t special[2];                                          // mass of the bins that hold several numbers, if others hold one
    uint64_t before, through;                                     // answers
    uint32_t held, bin, ahead, index;
};

// What lies before the thread's v in the workgroup, and all of it.
template <int THREADS, typename V>
__device__ __forceinline__ V before_thread(V v, V* sums, V& all) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    V upto = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const V other = (V)__shfl_up((unsigned long long)upto, o);
        if (lane >= (uint32_t)o) upto += other;
    }
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

enum Question { kCount, kMass, kValue };                          // at which place do count or mass reach a number, or logits a value

template <typename T, int THREADS>
struct Row {
    static constexpr uint32_t E = Pieces<T>::E;
    using Piece = typename Pieces<T>::Piece;
    static constexpr uint32_t kOwn = kBins / THREADS;             // bins of a thread
    SampleLds<THREADS>& s;
    const T* z;
    uint32_t vocab;
    Masses masses;
    Bins bins;
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

    // Gathers the logits from lo to hi (kList of them at most) as ranks; returns how many there are.
    __device__ uint32_t gather(float lo, float hi) {
        __syncthreads();
        if (threadIdx.x == 0) s.held = 0;
        __syncthreads();
        stream([&](const float(&v)[E], uint32_t at) {
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
    __device__ void settle(uint32_t n, uint64_t before) {
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t mine = s.list[i];
            uint32_t place = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < n; ++j) place += s.list[j] > mine ? 1u : 0u;
            s.sorted[place] = mine;
        }
        __syncthreads();
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
    __device__ uint64_t list_mass(uint32_t n, uint64_t before, uint64_t t) {
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
    __device__ uint64_t list_value(uint32_t n, uint64_t before, double d) {
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

    // The column of the nth (from 1) logit that equals `value`: each wave counts those of a stretch of the row.
    __device__ void find_nth(float value, uint64_t nth) {
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

    // Logits that are all `value`, n of them (kValue), behind `before`.
    __device__ uint64_t among_equals(Question q, float value, uint64_t n, uint64_t before, uint64_t t, double d, bool pick) {
        const uint64_t mass = masses(value);
        if (q == kValue) return before + ((double)value - masses.max >= d ? n * mass : 0);
        const uint64_t nth = q == kCount ? t : (t - before + mass - 1) / mass;
        if (pick) find_nth(value, nth);
        return before + nth * mass;
    }

    // The answer among the logits from lo to hi: the mass through the place where their count (kCount) or the mass, that of logits before them
    // included (kMass), reaches t, or through the last with z - max >= d (kValue).
    __device__ uint64_t through(Question q, float lo, float hi, uint64_t before, uint64_t t, double d, bool pick) {
        for (;;) {
            const uint32_t n = gather(lo, hi);
            if (n <= kList) {
                settle(n, before);
                if (q == kValue) return list_value(n, before, d);
                if (q == kMass) return list_mass(n, before, t);
                return s.upto[t - 1];
            }
            if (lo == hi) return among_equals(q, lo, n, before, t, d, pick);
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
            stream([&](const float(&v)[E], uint32_t at) {
#pragma unroll
                for (uint32_t e = 0; e < E; ++e)
                    if (v[e] >= lo && v[e] <= hi && at + e < vocab) {
                        const uint32_t part = (first - logit_key(v[e])) >> shift;
                        atomicAdd(&s.part_count[part], 1u);
                        atomicAdd(reinterpret_cast<unsigned long long*>(&s.part_mass[part]), (unsigned long long)masses(v[e]));
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
                float border = (float)(masses.max + d);
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
};

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) sample_kernel(SampleShape a) {
    constexpr bool kSingle = std::is_same_v<T, __bf16>;           // a bin is a number
    constexpr uint32_t E = Pieces<T>::E, kOwn = kBins / THREADS;
    __shared__ SampleLds<THREADS> s;
    const uint64_t row = a.row0 + blockIdx.x;
    Row<T, THREADS> r{s, static_cast<const T*>(a.z) + row * a.z_ld, (uint32_t)a.vocab, {}, {}, 0.f};
    float temperature = a.each.temperature_dev ? a.each.temperature_dev[row] : a.temperature;
    const int32_t top_k = a.each.top_k_dev ? a.each.top_k_dev[row] : a.top_k;
    const float top_p = a.each.top_p_dev ? a.each.top_p_dev[row] : a.top_p, min_p = a.each.min_p_dev ? a.each.min_p_dev[row] : a.min_p;
    uint32_t k = top_k > 0 && (uint32_t)top_k < r.vocab ? (uint32_t)top_k : 0;
    if (!(temperature >= __FLT_MIN__ && temperature < kInf)) {    // the largest logit
        temperature = 1.f;
        k = 1;
    }
    const bool by_mass = top_p < 1.f;

    // the largest
    float max = -kInf;
    r.stream([&](const float(&v)[E], uint32_t) { max = max_or_nan(max, largest_of(v)); });
    max = over_lanes<64>(max, [](float x, float y) { return max_or_nan(x, y); });
    if ((threadIdx.x & 63) == 0) s.most[threadIdx.x / 64] = max;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) max = max_or_nan(max, s.most[w]);
    if (max != max || max == -kInf) {                             // no answer
        if (threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = max;
        }
        return;
    }
    const bool infinite = max == kInf, by_value = min_p > 0.f && !infinite;                // (infinite ones are alike)
    const double t64 = (double)temperature;
    r.masses.max = (double)max;
    r.masses.scale = 1.44269504088896340736 / t64;
    r.masses.least = infinite ? 0.0 : -1000.0;
    r.masses.bits = 62 - (r.vocab > 1 ? 32 - __builtin_clz(r.vocab - 1) : 0);
    if (r.masses.bits > 51) r.masses.bits = 51;
    r.bins = bins_of(max, temperature);
    // below: masses of less than half of a unit.  (In 32 bits: off by less than what one unit more of the exponent allows for.)
    r.least = infinite ? kInf : fmaxf((float)((double)max - (r.masses.bits + 2) * 0.69314718055994530942 * t64 - fabs((double)max) * 0x1p-20), -__FLT_MAX__);
    const double border = !by_value ? -kInf : t64 * log((double)(min_p < 1.f ? min_p : 1.f));    // of z - max
    const float u = a.u[row];
    const uint64_t u64 = !(u > 0.f) ? 0 : u >= 1.f ? ~0ull : (uint64_t)((double)u * 0x1p64);
    // what the first logits must reach for top_p of S
    auto share = [&](uint64_t sum) {
        if (!(top_p > 0.f)) return (uint64_t)1;
        const uint64_t p64 = (uint64_t)((double)top_p * 0x1p64), low = p64 * sum;
        const uint64_t t = __umul64hi(p64, sum) + (low ? 1 : 0);
        return t ? t : (uint64_t)1;
    };
    auto answer = [&](uint64_t sum) {                             // s.index is the token's
        if (threadIdx.x != 0) return;
        const uint32_t index = s.index;
        a.token[row] = (int32_t)index;
        const double y = infinite ? 0.0 : ((double)(float)r.z[index] - (double)max) / t64;
        if (a.logp) a.logp[row] = (float)(y - log(ldexp((double)sum, -r.masses.bits)));
    };
    // everything that matters is in the list
    auto answer_from_list = [&](uint32_t n) {
        r.settle(n, 0);
        uint64_t sum = s.upto[k && k < n ? k - 1 : n - 1];
        if (by_mass) sum = r.list_mass(n, 0, share(sum));
        if (by_value) {
            const uint64_t kept = r.list_value(n, 0, border);
            sum = kept < sum ? kept : sum;
        }
        (void)r.list_mass(n, 0, __umul64hi(u64, sum) + 1);
        answer(sum);
    };
    if (r.vocab <= kList) return answer_from_list(r.gather(r.least, kInf));

    // counts of the bins
    uint32_t k_bin = 0, k_left = 0;                               // the bin of the k-th logit, and the how-manieth of it that is
    uint32_t count_before = 0, held = 0;
    if (kSingle || k) {
        for (uint32_t i = threadIdx.x; i < kBins; i += THREADS) s.count[i] = 0;
        if (threadIdx.x < 2) s.special[threadIdx.x] = 0;
        __syncthreads();
        r.stream([&](const float(&v)[E], uint32_t) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (v[e] >= r.least) {
                    const uint32_t bin = r.bins(v[e]);
                    atomicAdd(&s.count[bin], 1u);
                    if (kSingle && !r.bins.single(bin))
                        atomicAdd(reinterpret_cast<unsigned long long*>(&s.special[bin == kBins - 1]), (unsigned long long)r.masses(v[e]));
                }
        });
        __syncthreads();
        uint32_t own = 0;
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) own += s.count[threadIdx.x * kOwn + i];
        count_before = before_thread<THREADS>(own, s.counts, held);
        if (k >= held) k = 0;
        if (k) {
            if (count_before < k && k <= count_before + own) {
                uint32_t upto = count_before;
                for (uint32_t i = 0; i < kOwn; ++i) {
                    const uint32_t here = s.count[threadIdx.x * kOwn + i];
                    if (k <= upto + here) {
                        s.bin = threadIdx.x * kOwn + i;
                        s.ahead = upto;
                        s.held = upto + here;
                        break;
                    }
                    upto += here;
                }
            }
            __syncthreads();
            k_bin = s.bin;
            k_left = k - s.ahead;
            const uint32_t above = s.held;
            __syncthreads();
            if (above <= kList) return answer_from_list(r.gather(r.bins.lowest(k_bin) > r.least ? r.bins.lowest(k_bin) : r.least, kInf));
            if (!kSingle && r.bins.lowest(k_bin) > r.least) r.least = r.bins.lowest(k_bin);
        }
    }
    // masses of the bins
    if constexpr (!kSingle) {
        for (uint32_t i = threadIdx.x; i < kBins; i += THREADS) s.mass[i] = 0;
        __syncthreads();
        r.stream([&](const float(&v)[E], uint32_t) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (v[e] >= r.least)
                    atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[r.bins(v[e])]), (unsigned long long)r.masses(v[e]));
        });
        __syncthreads();
    }
    auto mass_of = [&](uint32_t bin) -> uint64_t {
        if constexpr (kSingle) {
            if (!r.bins.single(bin)) return s.special[bin == kBins - 1];
            const uint32_t n = s.count[bin];
            return n ? n * r.masses(r.bins.number(bin)) : 0;
        } else {
            return s.mass[bin];
        }
    };
    uint64_t own = 0, sum;
#pragma unroll 1
    for (uint32_t i = 0; i < kOwn; ++i) own += mass_of(threadIdx.x * kOwn + i);
    const uint64_t mass_before = before_thread<THREADS>(own, s.sums, sum);
    // s.bin and s.before: the bin in which mass reaches t, or the given one, and the mass before it
    auto find = [&](bool given, uint32_t which, uint64_t t) {
        const bool mine = given ? which / kOwn == threadIdx.x : mass_before < t && t <= mass_before + own;
        if (mine) {
            uint64_t upto = mass_before;
            for (uint32_t i = threadIdx.x * kOwn;; ++i) {
                const uint64_t here = mass_of(i);
                if (given ? i == which : t <= upto + here) {
                    s.bin = i;
                    s.before = upto;
                    break;
                }
                upto += here;
            }
        }
        __syncthreads();
    };
    auto through = [&](Question q, uint64_t t, double d, bool pick) {
        const uint32_t bin = s.bin;
        const uint64_t before = s.before;
        __syncthreads();
        const float hi = r.bins.highest(bin), lo = r.bins.lowest(bin);
        if (kSingle && r.bins.single(bin)) {
            const float value = r.bins.number(bin);
            const uint32_t n = s.count[bin];
            if (!pick || n > kList) return r.among_equals(q, value, n, before, t, d, pick);
            return r.through(q, value, value, before, t, d, pick);
        }
        return r.through(q, lo > r.least ? lo : r.least, hi, before, t, d, pick);
    };
    if (k) {
        find(true, k_bin, 0);
        sum = through(kCount, k_left, 0.0, false);
    }
    if (by_mass) {
        const uint64_t t = share(sum);
        find(false, 0, t);
        sum = through(kMass, t, 0.0, false);
    }
    if (by_value) {
        const float at = (float)(r.masses.max + border);
        if (at >= r.least) {
            find(true, r.bins(at), 0);
            const uint64_t kept = through(kValue, 0, border, false);
            sum = kept < sum ? kept : sum;
        }
    }
    const uint64_t t = __umul64hi(u64, sum) + 1;
    find(false, 0, t);
    (void)through(kMass, t, 0.0, true);
    answer(sum);
}

template <typename T>
void launch_sample_of(const SampleArgs& args, hipStream_t stream) {
    SampleShape a{};
    static_cast<SampleArgs&>(a) = args;
    for (uint64_t r = 0; r < a.rows; r += kRowsOfLaunch) {
        a.row0 = r;
        const unsigned here = (unsigned)(a.rows - r < kRowsOfLaunch ? a.rows - r : kRowsOfLaunch);
        if (a.vocab <= 16384) hipLaunchKernelGGL((sample_kernel<T, 256>), dim3(here), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((sample_kernel<T, 512>), dim3(here), dim3(512), 0, stream, a);
    }
}

}  // namespace

uint64_t sample_work_bytes(const ds_sampling&) { return 0; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_sample_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
