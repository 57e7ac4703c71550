// The loss of a row of logits against a teacher's (index, logit) pairs, and its gradient (ds_distill).
//
// Bound by reading the logits once and writing their gradient once.  A row stays in the registers of its workgroup between the sum of exponentials
// and the gradient (up to 256 KB: 1024 threads of 64 registers); the threads' number follows the row's length.  A workgroup takes one row after the other,
// and asks for the next row's logits as it writes: 16 bytes of gradient, and the registers they came from wait for 16 bytes of logits.  Where rows
// are longer, or too few to fill the GPU, they are split: a first launch sums the parts, a second one reads the logits again and writes the gradient.  The
// second read comes out of the memory-side cache where the call's logits fit it (100 x 200003, bf16: 30 us), otherwise from memory: 4096 x 151936, bf16,
// 773 us, three passes of 1.2 GB at 4.8 TB/s; 2048 x 100000, fp32, 486 us.
//   4096 x 131072, bf16: 440 us, 4.9 TB/s in and out; 1023 x 50001, fp16: 49 us, 4.2, in two rows of each workgroup, the first of which is waited for.  The
// exponentials are made twice, which with their arguments is most of the instructions: of 16 bits there is no room to keep them.
//   The listed columns are written once more, after the dense part, by the thread that has the first of the entries with that index.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

constexpr uint64_t kRowsOfLaunch = 1u << 21;                      // a launch dimension holds fewer than 2^32 work-items

struct DistillShape : LogitsArgs {
    uint64_t row0;
    uint64_t rows_here;                                           // rows of the launch, from row0 on
    uint32_t parts;                                               // workgroups of a row
    uint64_t part_logits;                                         // a multiple of what a workgroup takes at a time
    float2* spreads;                                              // [row][part]
    float* listed;                                                // [row][k]: the student's logits at the listed columns
};

// What the teacher says about a row: entry j of thread j < k.
struct Teacher {
    uint32_t index;
    bool listed;                                                  // the index is a column
    float log_p, p, z;                                            // ln p, p and the student's logit there
    float mass;                                                   // sum of p
};

template <int WAVES>
__device__ __forceinline__ float workgroup_total(float v, float* sums) {
    v = total_over_lanes<64>(v);
    if (WAVES == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = v;
    __syncthreads();
    return total_over_lanes<WAVES>(sums[threadIdx.x & (WAVES - 1)]);
}

// k <= 256: the entries are the first four waves'.
__device__ __forceinline__ uint2 teacher_pair(const LogitsArgs& a, uint64_t row) {
    return threadIdx.x < a.k ? a.given[row * a.k + threadIdx.x] : make_uint2(~0u, 0u);
}
template <int WAVES>
__device__ Teacher read_teacher(const LogitsArgs& a, uint64_t row, uint2 pair, float z, float scale, float* sums) {
    Teacher e;
    e.index = pair.x;
    e.listed = pair.x < a.vocab;
    e.z = z;
    const float logit = __uint_as_float(pair.y);
    if (a.teacher_lse) {
        e.log_p = logit / a.temperature - a.teacher_lse[row];
    } else {
        const Spread s = workgroup_spread<WAVES>(e.listed ? spread_of(logit, scale) : kNoSpread, scale, sums);
        const LogSum l = log_sum(s, scale);
        e.log_p = (logit - l.from) / a.temperature - l.rest;
    }
    e.p = e.listed && logit != -__builtin_huge_valf() ? expf(e.log_p) : 0.f;
    e.mass = workgroup_total<WAVES>(e.p, sums);
    return e;
}

// The entry's share of the loss.
__device__ __forceinline__ float listed_term(const Teacher& e, LogSum l, float temperature, float weight) {
    if (e.p == 0.f) return 0.f;
    const float q = (e.z - l.from) / temperature;
    if (fabsf(q) != kInf || fabsf(e.z) == kInf) return weight * (e.p * (e.log_p - q + l.rest));
    // q is beyond fp32 (a mask of the lowest value, T < 1): weight p q may not be
    return weight * (e.p * (e.log_p + l.rest)) - weight * (2.f * e.p) / temperature * (0.5f * e.z - 0.5f * l.from);
}

// The row's entries in LDS.
struct Listed {
    uint32_t index[kMaxTop];
    float p[kMaxTop];
    uint32_t mixed;                                               // an index is not above the one before: some may be the same
};
__device__ __forceinline__ void keep_listed(const Teacher& e, uint32_t k, Listed& listed) {
    if (threadIdx.x == 0) listed.mixed = 0;
    if (threadIdx.x < k) {
        listed.index[threadIdx.x] = e.index;
        listed.p[threadIdx.x] = e.p;
    }
    __syncthreads();
    if (threadIdx.x && threadIdx.x < k && listed.index[threadIdx.x - 1] >= e.index) listed.mixed = 1;
}

// What a row's gradient is made of: dz = each 2^(exponent of z) - c (sum of the column's p).
struct Gradient {
    Exponents e;
    float each, c;
};
template <typename T>
__device__ __forceinline__ typename Pieces<T>::Piece gradient_piece(const Gradient& g, typename Pieces<T>::Piece z) {
    typename Pieces<T>::Piece out;
#pragma unroll
    for (uint32_t i = 0; i < Pieces<T>::E; ++i) out[i] = (T)(g.each * g.e((float)z[i]));
    return out;
}
// dz of the listed columns in [begin, end), when the dense part is written.
template <typename T>
__device__ __forceinline__ void write_listed(const Gradient& g, const Teacher& e, const Listed& listed, uint32_t k, uint64_t begin, uint64_t end, T* dz) {
    if (!e.listed || e.index < begin || e.index >= end) return;
    float all = e.p;
    if (listed.mixed) {
        all = 0.f;
#pragma unroll 8
        for (uint32_t i = 0; i < k; ++i) {
            if (listed.index[i] != e.index) continue;
            if (i < threadIdx.x) return;                          // the first of them writes
            all += listed.p[i];
        }
    }
    dz[e.index] = (T)(g.each * g.e(e.z) - g.c * all);
}

// A workgroup per row at a time, N 16-byte pieces of it in each thread's registers.
template <typename T, int THREADS, int N>
__global__ void __launch_bounds__(THREADS) distill_row_kernel(DistillShape a) {
    constexpr int WAVES = THREADS / 64;
    constexpr uint32_t E = Pieces<T>::E;
    using Piece = typename Pieces<T>::Piece;
    __shared__ float sums[2 * WAVES];
    __shared__ Listed listed;
    const float scale = kLog2e / a.temperature;
    const uint32_t vocab = (uint32_t)a.vocab, whole = vocab / E;   // pieces without the ragged end
    const bool rest = whole * E + threadIdx.x < vocab;            // the thread has a column of it
    u32x4 raw[N];                                                 // (bits: as numbers the compiler would keep them in fp32, twice as many registers)
    float last = -kInf;
    Piece nothing;
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) nothing[e] = (T)-kInf;
    auto load = [&](const T* z, int p) {
        raw[p] = __builtin_bit_cast(u32x4, nothing);
        if (p * THREADS + threadIdx.x < whole)                    // (an address for all, and the thread's 32 bits)
            raw[p] = __builtin_bit_cast(u32x4, *reinterpret_cast<const Piece*>(reinterpret_cast<const uint8_t*>(z) + p * (THREADS * 16) + threadIdx.x * 16u));
    };
    auto logits = [&](uint64_t r) { return static_cast<const T*>(a.z) + r * a.z_ld; };
    uint64_t row = a.row0 + blockIdx.x;
    const uint64_t end = a.row0 + a.rows_here;
    auto weight_of = [&](uint64_t r) { return a.weight ? a.weight[r] : 1.f; };
    float weight = row < end ? weight_of(row) : 0.f;
    if (weight != 0.f) {
#pragma unroll
        for (int p = 0; p < N; ++p) load(logits(row), p);
        if (rest) last = (float)logits(row)[whole * E + threadIdx.x];
    }
    for (; row < end; row += gridDim.x) {
        T* dz = a.dz ? static_cast<T*>(a.dz) + row * a.dz_ld : nullptr;
        const uint64_t next = row + gridDim.x;
        const float next_weight = next < end ? weight_of(next) : 0.f;
        Gradient g{{0.f, 0.f, false}, 0.f, 0.f};
        bool skip = weight == 0.f;                                // a padded token: its logits are not read
        Teacher teacher{};
        if (!skip) {
            const uint2 pair = teacher_pair(a, row);
            const float at_pair = pair.x < vocab ? (float)logits(row)[pair.x] : 0.f;
            teacher = read_teacher<WAVES>(a, row, pair, at_pair, scale, sums);
            keep_listed(teacher, a.k, listed);
            Spread s = kNoSpread;
#pragma unroll
            for (int p = 0; p < N; p += N > 1 ? 2 : 1) {          // as the pieces arrive
                constexpr int M = N > 1 ? 2 : 1;
                float v[M][E], most[M];
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    u32x4 bits = raw[p + m];
                    asm volatile("" : "+v"(bits), "+v"(s.sum));   // when the pieces before are done
                    const Piece piece = __builtin_bit_cast(Piece, bits);
#pragma unroll
                    for (uint32_t e = 0; e < E; ++e) v[m][e] = (float)piece[e];
                    most[m] = largest_of(v[m]);
                }
                add_logits(s, v, largest_of(most), scale);
            }
            s = join(s, spread_of(last, scale), scale);
            s = workgroup_spread<WAVES>(s, scale, sums);
            const LogSum l = log_sum(s, scale);
            if (a.loss) {
                const float terms = workgroup_total<WAVES>(listed_term(teacher, l, a.temperature, weight), sums);
                if (threadIdx.x == 0) a.loss[row] = teacher.mass == 0.f ? 0.f : terms;
            }
            g = {exponents(s.max, scale), weight / a.temperature * teacher.mass / s.sum, weight / a.temperature};
            skip = teacher.mass == 0.f;
        } else if (a.loss && threadIdx.x == 0) {
            a.loss[row] = 0.f;
        }
        const bool more = next_weight != 0.f;
        const T* z_next = logits(more ? next : row);
#pragma unroll
        for (int p = 0; p < N; ++p) {
            asm volatile("" : "+v"(raw[p]) : : "memory");         // one after the other: all exponentials at once would take as many registers again
            if (dz && p * THREADS + threadIdx.x < whole) {
                Piece out;
                if (skip) {
#pragma unroll
                    for (uint32_t e = 0; e < E; ++e) out[e] = (T)0.f;
                } else {
                    out = gradient_piece<T>(g, __builtin_bit_cast(Piece, raw[p]));
                }
                *reinterpret_cast<Piece*>(reinterpret_cast<uint8_t*>(dz) + p * (THREADS * 16) + threadIdx.x * 16u) = out;
            }
            if (more) load(z_next, p);
        }
        if (dz && rest) dz[whole * E + threadIdx.x] = skip ? (T)0.f : (T)(g.each * g.e(last));
        if (more && rest) last = (float)z_next[whole * E + threadIdx.x];
        __syncthreads();
        if (dz && !skip) write_listed(g, teacher, listed, a.k, 0, vocab, dz);
        weight = next_weight;
    }
}

constexpr int kPartThreads = 256, kPartWaves = kPartThreads / 64, kPartPieces = 4;

// First launch of split rows: the sum of a part, and in the workgroup of the first part the listed logits, while z is still whole (dz may take
// its place).
template <typename T>
__global__ void __launch_bounds__(kPartThreads) distill_sum_kernel(DistillShape a) {
    constexpr uint32_t E = Pieces<T>::E, kStretch = kPartThreads * kPartPieces * E;
    using Piece = typename Pieces<T>::Piece;
    __shared__ float sums[2 * kPartWaves];
    const uint64_t row = a.row0 + blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    if (a.weight && a.weight[row] == 0.f) return;
    const float scale = kLog2e / a.temperature;
    const uint64_t begin = (uint64_t)blockIdx.y * a.part_logits, end = begin + a.part_logits < a.vocab ? begin + a.part_logits : a.vocab;
    Spread s = kNoSpread;
    for (uint64_t at = begin; at < end; at += kStretch) {
        float v[kPartPieces][E], most[kPartPieces];
        const uint64_t mine = at + (uint64_t)threadIdx.x * E;
        if (at + kStretch <= end) {
            Piece raw[kPartPieces];
#pragma unroll
            for (int p = 0; p < kPartPieces; ++p) raw[p] = *reinterpret_cast<const Piece*>(z + mine + (uint64_t)p * kPartThreads * E);
#pragma unroll
            for (int p = 0; p < kPartPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) v[p][e] = (float)raw[p][e];
        } else {
#pragma unroll
            for (int p = 0; p < kPartPieces; ++p)
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) {
                    const uint64_t c = mine + (uint64_t)p * kPartThreads * E + e;
                    v[p][e] = c < end ? (float)z[c] : -kInf;
                }
        }
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p) most[p] = largest_of(v[p]);
        add_logits(s, v, largest_of(most), scale);
    }
    s = workgroup_spread<kPartWaves>(s, scale, sums);
    if (threadIdx.x == 0) a.spreads[row * a.parts + blockIdx.y] = make_float2(s.max, s.sum);
    if (blockIdx.y != 0 || threadIdx.x >= a.k) return;
    const uint2 pair = teacher_pair(a, row);
    a.listed[row * a.k + threadIdx.x] = pair.x < a.vocab ? (float)z[pair.x] : 0.f;
}

// Second launch: the loss, and the gradient of a part.
template <typename T>
__global__ void __launch_bounds__(kPartThreads) distill_part_kernel(DistillShape a) {
    constexpr uint32_t E = Pieces<T>::E, kStretch = kPartThreads * kPartPieces * E;
    using Piece = typename Pieces<T>::Piece;
    __shared__ float sums[2 * kPartWaves];
    __shared__ Listed listed;
    const uint64_t row = a.row0 + blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    T* dz = a.dz ? static_cast<T*>(a.dz) + row * a.dz_ld : nullptr;
    const float scale = kLog2e / a.temperature, weight = a.weight ? a.weight[row] : 1.f;
    const uint64_t begin = (uint64_t)blockIdx.y * a.part_logits, end = begin + a.part_logits < a.vocab ? begin + a.part_logits : a.vocab;
    Piece raw[kPartPieces];
    auto load = [&](uint64_t at) {
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p) {
            const uint64_t col = at + (uint64_t)(p * kPartThreads + threadIdx.x) * E;
            if (col + E <= end) raw[p] = *reinterpret_cast<const Piece*>(z + col);
            else
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) raw[p][e] = col + e < end ? z[col + e] : (T)0.f;
        }
    };
    // all that is read without knowing more is asked for at once
    if (dz && weight != 0.f) load(begin);
    const uint2 pair = teacher_pair(a, row);
    const float z_pair = threadIdx.x < a.k ? a.listed[row * a.k + threadIdx.x] : 0.f;
    const float2 of_part = threadIdx.x < a.parts ? a.spreads[row * a.parts + threadIdx.x] : make_float2(-kInf, 0.f);   // (parts <= 256)
    bool skip = weight == 0.f;
    Teacher teacher{};
    Gradient g{{0.f, 0.f, false}, 0.f, 0.f};
    if (!skip) {
        teacher = read_teacher<kPartWaves>(a, row, pair, z_pair, scale, sums);
        keep_listed(teacher, a.k, listed);
        Spread s = {of_part.x, of_part.y};
        s = workgroup_spread<kPartWaves>(s, scale, sums);
        const LogSum l = log_sum(s, scale);
        skip = teacher.mass == 0.f;
        if (a.loss && blockIdx.y == 0) {
            const float terms = workgroup_total<kPartWaves>(listed_term(teacher, l, a.temperature, weight), sums);
            if (threadIdx.x == 0) a.loss[row] = skip ? 0.f : terms;
        }
        g = {exponents(s.max, scale), weight / a.temperature * teacher.mass / s.sum, weight / a.temperature};
    } else if (a.loss && blockIdx.y == 0 && threadIdx.x == 0) {
        a.loss[row] = 0.f;
    }
    if (!dz) return;
    for (uint64_t at = begin; at < end; at += kStretch) {
        if (at > begin && !skip) load(at);
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p) {
            const uint64_t col = at + (uint64_t)(p * kPartThreads + threadIdx.x) * E;
            if (col >= end) break;
            Piece out;
            const bool whole = col + E <= end;
            if (skip) {
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) out[e] = (T)0.f;
            } else {
                out = gradient_piece<T>(g, raw[p]);
            }
            if (whole) *reinterpret_cast<Piece*>(dz + col) = out;
            else
#pragma unroll
                for (uint32_t e = 0; e < E; ++e)
                    if (col + e < end) dz[col + e] = out[e];
        }
    }
    __syncthreads();
    if (!skip) write_listed(g, teacher, listed, a.k, begin, end, dz);
}

constexpr uint64_t kRowBytes = 1024 * 16 * 16;                    // of the longest row that stays in registers

// Rows that stay whole have parts = 0.
void distill_plan(uint64_t rows, uint64_t vocab, uint64_t size, uint32_t& parts, uint64_t& part_logits) {
    parts = 0;
    part_logits = vocab;
    // One launch where it holds up: rows 8 x 32003 f32 9.2 us, and 4.0 + 5.5 split; 1 x 65536 bf16 11.0 and 3.6 + 5.5; 1 x 131072 bf16 18.0 and 3.4 + 5.4; 64 x
    // 131072 22.5 and 7.0 + 9.5; 200 x 131072 27.9 and 13.1 + 20.1.
    if (vocab * size <= kRowBytes && (rows >= 128 || vocab * size <= kRowBytes / 2)) return;
    const uint64_t stretch = kPartThreads * kPartPieces * (16 / size), stretches = (vocab + stretch - 1) / stretch;
    uint64_t p = rows >= 1024 ? 1 : 1024 / rows;
    if (p > stretches) p = stretches;
    if (p > 256) p = 256;
    const uint64_t each = (stretches + p - 1) / p;
    part_logits = each * stretch;
    parts = (uint32_t)((stretches + each - 1) / each);
}

// Few threads with much of a row each, so that a compute unit has several rows under way: 4096 x 32000 bf16 with 256 threads 113 us, 512 136, 1024 233;
// 1023 x 50001 f16 with 512 49, 1024 74.  As many workgroups as run at once, each with rows of its own (RESIDENT a compute unit): 1023 x 50001 49 us, and 54 with
// one for each row.  Where a compute unit holds one row it gains nothing, and rows of weight 0 leave some with less to do than others (RESIDENT = 0: one for
// each row): 4096 x 131072 bf16 439 us, and 471.
template <typename T, int THREADS, int N, int RESIDENT>
void launch_rows(const DistillShape& a, unsigned here, hipStream_t stream) {
    constexpr unsigned most = 256 * RESIDENT;
    hipLaunchKernelGGL((distill_row_kernel<T, THREADS, N>), dim3(RESIDENT && here > most ? most : here), dim3(THREADS), 0, stream, a);
}

template <typename T>
void launch_distill_of(const LogitsArgs& args, hipStream_t stream) {
    DistillShape a{};
    static_cast<LogitsArgs&>(a) = args;
    distill_plan(a.rows, a.vocab, sizeof(T), a.parts, a.part_logits);
    a.spreads = static_cast<float2*>(a.work);
    a.listed = reinterpret_cast<float*>(a.spreads + a.rows * a.parts);
    for (uint64_t r = 0; r < a.rows; r += kRowsOfLaunch) {
        a.row0 = r;
        const unsigned here = (unsigned)(a.rows - r < kRowsOfLaunch ? a.rows - r : kRowsOfLaunch);
        a.rows_here = here;
        if (a.parts) {
            hipLaunchKernelGGL(distill_sum_kernel<T>, dim3(here, a.parts), dim3(kPartThreads), 0, stream, a);
            hipLaunchKernelGGL(distill_part_kernel<T>, dim3(here, a.parts), dim3(kPartThreads), 0, stream, a);
            continue;
        }
        const uint64_t bytes = a.vocab * sizeof(T);
        if (bytes <= 4096) launch_rows<T, 256, 1, 7>(a, here, stream);
        else if (bytes <= 8192) launch_rows<T, 256, 2, 7>(a, here, stream);
        else if (bytes <= 16384) launch_rows<T, 256, 4, 6>(a, here, stream);
        else if (bytes <= 32768) launch_rows<T, 256, 8, 5>(a, here, stream);
        else if (bytes <= 65536) launch_rows<T, 256, 16, 4>(a, here, stream);
        else if (bytes <= 131072) launch_rows<T, 512, 16, 2>(a, here, stream);
        else launch_rows<T, 1024, 16, 0>(a, here, stream);
    }
}

}  // namespace

uint64_t distill_work_bytes(const ds_logits& l) {
    uint32_t parts;
    uint64_t part_logits;
    distill_plan(l.rows, l.vocab, l.dtype == DS_F32 ? 4 : 2, parts, part_logits);
    return parts ? l.rows * (parts * sizeof(float2) + (uint64_t)l.k * sizeof(float)) : 0;
}

hipError_t launch_distill(const LogitsArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_distill_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
