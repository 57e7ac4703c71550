// The loss of a row of logits against a teacher's (index, logit) pairs, and its gradient (ds_distill).
//
// Bound by reading the logits once and writing their gradient once.  A row stays in the registers of its workgroup between the sum of exponentials
// and the gradient (up to 256 KB: 1024 threads of 64 registers); the threads' number follows the row's length.  A wave's reduction and two barriers
// join the threads' sums.  Where rows are longer, or too few to fill the GPU, they are split: a first launch sums the parts, a second one
// reads the logits again (out of the memory-side cache, mostly) and writes the gradient.
//   The listed columns are written once more, after the dense part, by the thread that has the first of the entries with that index.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

constexpr uint64_t kRowsOfLaunch = 1u << 21;                      // a launch dimension holds fewer than 2^32 work-items

struct DistillShape : LogitsArgs {
    uint64_t row0;
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
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    if (WAVES == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < WAVES; ++w) v += sums[w];
    return v;
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
        const Spread s = workgroup_spread<WAVES>(e.listed ? spread_of(logit) : kNoSpread, scale, sums);
        e.log_p = (logit - reference(s.max)) / a.temperature - kLn2 * log2f(s.sum);
    }
    e.p = e.listed && logit != -__builtin_huge_valf() ? expf(e.log_p) : 0.f;
    e.mass = workgroup_total<WAVES>(e.p, sums);
    return e;
}

__device__ __forceinline__ float listed_term(const Teacher& e, float top, float temperature) {
    return e.p != 0.f ? e.p * (e.log_p - (e.z - top) / temperature) : 0.f;
}

// dz of the listed columns in [begin, end): each from the thread that holds the first of its entries.  Called when the dense part is written.
// index, prob: 256 of LDS each, which hold the entries since the last barrier.
template <typename T>
__device__ void write_listed(const Teacher& e, uint32_t k, const uint32_t* index, const float* prob, float each, float c, float top, float scale,
                             uint64_t begin, uint64_t end, T* dz) {
    if (!e.listed || e.index < begin || e.index >= end) return;
    float all = 0.f;
    bool mine = true;
    for (uint32_t i = 0; i < k; ++i)
        if (index[i] == e.index) {
            mine = mine && i >= threadIdx.x;
            all += prob[i];
        }
    if (mine) dz[e.index] = (T)(each * power2((e.z - top) * scale) - c * all);
}

template <typename T>
struct Pieces {
    static constexpr uint32_t E = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// A workgroup per row, N 16-byte pieces of it in each thread's registers.
template <typename T, int THREADS, int N>
__global__ void __launch_bounds__(THREADS) distill_row_kernel(DistillShape a) {
    constexpr int WAVES = THREADS / 64;
    constexpr uint32_t E = Pieces<T>::E;
    using Piece = typename Pieces<T>::Piece;
    __shared__ float sums[2 * WAVES];
    __shared__ uint32_t index[kMaxTop];
    __shared__ float prob[kMaxTop];
    const uint64_t row = a.row0 + blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    T* dz = a.dz ? static_cast<T*>(a.dz) + row * a.dz_ld : nullptr;
    const float scale = kLog2e / a.temperature, weight = a.weight ? a.weight[row] : 1.f;
    const uint32_t vocab = (uint32_t)a.vocab, whole = vocab / E;   // pieces without the ragged end
    const T zero = (T)0.f;

    if (weight == 0.f) {                                          // a padded token: its logits are not read
        if (a.loss && threadIdx.x == 0) a.loss[row] = 0.f;
        if (!dz) return;
        Piece none;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) none[e] = zero;
        for (uint32_t p = threadIdx.x; p < whole; p += THREADS) *reinterpret_cast<Piece*>(dz + (uint64_t)p * E) = none;
        for (uint32_t v = whole * E + threadIdx.x; v < vocab; v += THREADS) dz[v] = zero;
        return;
    }
    const uint2 pair = teacher_pair(a, row);
    const float listed = pair.x < vocab ? (float)z[pair.x] : 0.f;
    u32x4 raw[N];                                                 // (bits: as numbers the compiler would keep them in fp32, twice as many registers)
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const uint32_t at = p * THREADS + threadIdx.x;
        Piece v;
        if (at < whole) v = *reinterpret_cast<const Piece*>(z + (uint64_t)at * E);
        else {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) v[e] = at == whole && at * E + e < vocab ? z[at * E + e] : (T)-__builtin_huge_valf();
        }
        raw[p] = __builtin_bit_cast(u32x4, v);
    }
    const Teacher teacher = read_teacher<WAVES>(a, row, pair, listed, scale, sums);
    if (threadIdx.x < a.k) {
        index[threadIdx.x] = teacher.index;
        prob[threadIdx.x] = teacher.p;
    }
    Spread s = kNoSpread;
#pragma unroll
    for (int p = 0; p < N; ++p) {                                 // as the pieces arrive
        const Piece v = __builtin_bit_cast(Piece, raw[p]);
        float m = s.max;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) m = fmaxf(m, (float)v[e]);
        const float r = reference(m);
        float total = s.sum == 0.f ? 0.f : s.sum * power2((reference(s.max) - r) * scale);
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) total += power2(((float)v[e] - r) * scale);
        s = {m, total};
        asm volatile("" : "+v"(raw[p]));
    }
    s = workgroup_spread<WAVES>(s, scale, sums);
    const float top = reference(s.max), log_sum = kLn2 * log2f(s.sum);
    if (a.loss) {
        const float terms = workgroup_total<WAVES>(listed_term(teacher, top, a.temperature), sums);
        if (threadIdx.x == 0) a.loss[row] = teacher.mass == 0.f ? 0.f : weight * (terms + teacher.mass * log_sum);
    }
    if (!dz) return;
    const float c = weight / a.temperature, each = c * teacher.mass / s.sum;
    const bool skip = teacher.mass == 0.f;
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const uint32_t at = p * THREADS + threadIdx.x;
        const Piece v = __builtin_bit_cast(Piece, raw[p]);
        Piece out;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) out[e] = skip ? zero : (T)(each * power2(((float)v[e] - top) * scale));
        if (at < whole) *reinterpret_cast<Piece*>(dz + (uint64_t)at * E) = out;
        else if (at == whole) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (at * E + e < vocab) dz[at * E + e] = out[e];
        }
    }
    __syncthreads();
    if (!skip) write_listed(teacher, a.k, index, prob, each, c, top, scale, 0, vocab, dz);
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
        Piece raw[kPartPieces];
        const uint64_t mine = at + (uint64_t)threadIdx.x * E;
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p) {
            const uint64_t c = mine + (uint64_t)p * kPartThreads * E;
            if (c + E <= end) raw[p] = *reinterpret_cast<const Piece*>(z + c);
            else
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) raw[p][e] = c + e < end ? z[c + e] : (T)-__builtin_huge_valf();
        }
        float m = s.max;
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p)
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) m = fmaxf(m, (float)raw[p][e]);
        const float r = reference(m);
        float total = 0.f;
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p)
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) total += power2(((float)raw[p][e] - r) * scale);
        if (s.sum != 0.f) total = fmaf(s.sum, exp2f((reference(s.max) - r) * scale), total);
        s = {m, total};
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
    __shared__ uint32_t index[kMaxTop];
    __shared__ float prob[kMaxTop];
    const uint64_t row = a.row0 + blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    T* dz = a.dz ? static_cast<T*>(a.dz) + row * a.dz_ld : nullptr;
    const float scale = kLog2e / a.temperature, weight = a.weight ? a.weight[row] : 1.f;
    const uint64_t begin = (uint64_t)blockIdx.y * a.part_logits, end = begin + a.part_logits < a.vocab ? begin + a.part_logits : a.vocab;
    bool skip = weight == 0.f;
    Teacher teacher{};
    float top = 0.f, c = 0.f, each = 0.f;
    if (!skip) {
        teacher = read_teacher<kPartWaves>(a, row, teacher_pair(a, row), threadIdx.x < a.k ? a.listed[row * a.k + threadIdx.x] : 0.f, scale, sums);
        if (threadIdx.x < a.k) {
            index[threadIdx.x] = teacher.index;
            prob[threadIdx.x] = teacher.p;
        }
        Spread s = kNoSpread;
        for (uint32_t p = threadIdx.x; p < a.parts; p += kPartThreads) {
            const float2 v = a.spreads[row * a.parts + p];
            s = join(s, Spread{v.x, v.y}, scale);
        }
        s = workgroup_spread<kPartWaves>(s, scale, sums);
        top = reference(s.max);
        c = weight / a.temperature;
        each = c * teacher.mass / s.sum;
        skip = teacher.mass == 0.f;
        if (a.loss && blockIdx.y == 0) {
            const float terms = workgroup_total<kPartWaves>(listed_term(teacher, top, a.temperature), sums);
            if (threadIdx.x == 0) a.loss[row] = skip ? 0.f : weight * (terms + teacher.mass * (kLn2 * log2f(s.sum)));
        }
    } else if (a.loss && blockIdx.y == 0 && threadIdx.x == 0) {
        a.loss[row] = 0.f;
    }
    if (!dz) return;
    for (uint64_t at = begin; at < end; at += kStretch) {
        const uint64_t mine = at + (uint64_t)threadIdx.x * E;
#pragma unroll
        for (int p = 0; p < kPartPieces; ++p) {
            const uint64_t col = mine + (uint64_t)p * kPartThreads * E;
            if (col >= end) break;
            Piece raw, out;
            const bool whole = col + E <= end;
            if (skip) {
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) out[e] = (T)0.f;
            } else {
                if (whole) raw = *reinterpret_cast<const Piece*>(z + col);
                else
#pragma unroll
                    for (uint32_t e = 0; e < E; ++e) raw[e] = col + e < end ? z[col + e] : (T)0.f;
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) out[e] = (T)(each * power2(((float)raw[e] - top) * scale));
            }
            if (whole) *reinterpret_cast<Piece*>(dz + col) = out;
            else
#pragma unroll
                for (uint32_t e = 0; e < E; ++e)
                    if (col + e < end) dz[col + e] = out[e];
        }
    }
    __syncthreads();
    if (!skip) write_listed(teacher, a.k, index, prob, each, c, top, scale, begin, end, dz);
}

constexpr uint64_t kRowBytes = 1024 * 16 * 16;                    // of the longest row that stays in registers

// Rows that stay whole have parts = 0.
void distill_plan(uint64_t rows, uint64_t vocab, uint64_t size, uint32_t& parts, uint64_t& part_logits) {
    parts = 0;
    part_logits = vocab;
    if (vocab * size <= kRowBytes && (rows >= 128 || vocab * size <= 16384)) return;
    const uint64_t stretch = kPartThreads * kPartPieces * (16 / size), stretches = (vocab + stretch - 1) / stretch;
    uint64_t p = rows >= 1024 ? 1 : 1024 / rows;
    if (p > stretches) p = stretches;
    if (p > 256) p = 256;
    const uint64_t each = (stretches + p - 1) / p;
    part_logits = each * stretch;
    parts = (uint32_t)((stretches + each - 1) / each);
}

template <typename T, int THREADS, int N>
void launch_rows(const DistillShape& a, unsigned here, hipStream_t stream) {
    hipLaunchKernelGGL((distill_row_kernel<T, THREADS, N>), dim3(here), dim3(THREADS), 0, stream, a);
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
        if (a.parts) {
            hipLaunchKernelGGL(distill_sum_kernel<T>, dim3(here, a.parts), dim3(kPartThreads), 0, stream, a);
            hipLaunchKernelGGL(distill_part_kernel<T>, dim3(here, a.parts), dim3(kPartThreads), 0, stream, a);
            continue;
        }
        const uint64_t bytes = a.vocab * sizeof(T);
        if (bytes <= 4096) launch_rows<T, 256, 1>(a, here, stream);
        else if (bytes <= 8192) launch_rows<T, 256, 2>(a, here, stream);
        else if (bytes <= 16384) launch_rows<T, 256, 4>(a, here, stream);
        else if (bytes <= 32768) launch_rows<T, 256, 8>(a, here, stream);
        else if (bytes <= 65536) launch_rows<T, 512, 8>(a, here, stream);
        else if (bytes <= 131072) launch_rows<T, 1024, 8>(a, here, stream);
        else launch_rows<T, 1024, 16>(a, here, stream);
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
