// Products with a matrix that is held as messages (ds_product): y = x M^T, M's rows as 4-bit codes with a scale per block.
//
// Reading the message, 0.53 bytes a weight, is what cannot be done without, and leaves time for some four vector instructions a weight's
// share of a lane.  16-bit types: x goes into matrix instructions as it is, a code as 0.5 + q / 32 (dsq_codes.h), which takes one vector instruction, and
// what that is too large by is where sums start: -47/64 sum x of a block.  Products are exact and sums are fp32; a block's scale multiplies its sum.
//   fp32: x is made of bytes, and the products are integers: per token and 128 columns ("chunk"; 64 where a block is 64), x = 2^e v with integers v of 32
// bits, written as four signed bytes, which an i8 matrix instruction takes as rows of their own, against codes as bytes.  All sums inside a chunk are exact; 15 sum v,
// which takes codes 0 .. 15 to 2 code - 15, is where they start.  What is rounded is v: by 2^-31 of the largest |x| next to it at most, of which
// y has 1/15 of the scale or more: no rounding is above 2^-27 of what that one contributes.
//   A wave takes 16 (or 32) rows and a chunk at a time: lane (n, j) = (l % 16, l / 16) holds 32 codes of row n and the scale of its block, which is
// one factor for all of the lane's results.  x lies in LDS in the order in which codes come out of a word.
//   Three kernels.  One token: product_one_kernel.  Up to 16 tokens (8 for fp32), where reading codes is most of the work:
// product_tiles_kernel, whose workgroups lay out x themselves.  More tokens: product_kernel; a launch before lays x out once, in work_dev,
// and codes go straight into registers, which leaves LDS to x.  Measured, us, product_tiles_kernel : product_kernel: 2 x 65536 x 4096,
// bf16, 30.7 : 64.4; 16 x 4096 x 16384, fp16, 18.3 : 23.7; 16 x 65536 x 4096, bf16, 40.0 : 66.2; 8 x 2048 x 2048, fp32, 7.6 : 9.6; 4 x 16384 x 4096, fp32,
// 17.3 : 20.5; one launch of product_tiles_kernel after the other: 17 x 65536 x 4096, bf16, 70.2 : 55.5; 32 tokens 79.0 : 56.2; 16 x 16384 x 4096, fp32, 38.6 : 21.7.
//   Where there are too few rows for the GPU, workgroups split the columns, too, and one more launch adds their sums.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_message_reads.h"

namespace dsq {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64, kChunk = 128;   // of a workgroup; columns a wave takes at a time
constexpr uint64_t kGroupsOfLaunch = 1u << 22;                    // a launch dimension holds fewer than 2^32 work-items

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// What a matrix instruction's 16 rows are: tokens, or for fp32 four digits of four tokens.
template <typename T>
constexpr int kTokenRows = sizeof(T) == 4 ? 4 : 1;
template <typename T>
using Coded = std::conditional_t<sizeof(T) == 4, __bf16, T>;        // (codes as a matrix instruction's numbers: of 16-bit types)
template <typename T>
constexpr int kTileTokens = 16 / kTokenRows<T>;                   // tokens of a matrix instruction
template <typename T>
constexpr int kMostTiles = sizeof(T) == 4 ? 8 : 4;                // of a launch
template <typename T>
constexpr int kFewTiles = sizeof(T) == 4 ? 2 : 1;                 // of product_tiles_kernel
template <typename T>
constexpr uint64_t kTokens = kMostTiles<T> * kTileTokens<T>;      // of a launch
// x of fp32 as integers: |v| <= 127 (2^24 + 2^16 + 2^8 + 1), below 2^31, and as a number of fp32.
constexpr int kExponent = 30;
constexpr float kMostDigits = 2139062016.f;
constexpr int kRowTiles = 2;                                      // of 16 rows, of a wave of product_kernel

struct ProductPlan {
    uint32_t parts, part_chunks;                                  // workgroups that split the columns, and the chunks (product_tiles_kernel: stages) of each
    uint32_t row_waves, wave_rows;                                // one token: waves side by side, the other kWaves / row_waves split the columns; rows of a wave
};

struct ProductShape : ProductArgs {
    ProductPlan plan;
    uint64_t row0;
    const uint8_t* panel;                                         // x laid out, one record per chunk (see Record), or nullptr
    float* partial;                                               // parts x tokens x rows, or nullptr
};

// One chunk of x.  16-bit types: x in the order of codes, [word of a lane][j][token][8 columns], and what products start from, -kCentre sum x, [block][token].
// fp32: the digits, [matrix instruction][j][row][16 columns] with digit d of token t in row 4 t + d; where the products start, -15 times the digits' sum,
// [block][row]; and per token what v counts, over 2^kExponent.  (Two blocks where a block is 64 columns.)  Rows of no token hold anything.
template <typename T, int TT, bool NARROW>
struct Record {
    static constexpr uint32_t H = NARROW ? 2 : 1, rows = 16 * TT;
    static constexpr uint32_t x_bytes = (sizeof(T) == 4 ? 128 : 256) * rows, sums = H * rows * 4;
    static constexpr uint32_t units = sizeof(T) == 4 ? H * rows : 0, bytes = x_bytes + sums + units;
    static_assert(bytes % 16 == 0);
    __device__ static u32x4* x(uint8_t* r) { return reinterpret_cast<u32x4*>(r); }
    __device__ static void* start(uint8_t* r) { return r + x_bytes; }
    __device__ static float* unit(uint8_t* r) { return reinterpret_cast<float*>(r + x_bytes + sums); }
};

// One weight after the other, as the formula has it: for a result that is not finite.  A thread goes through the row by itself, up to the first NaN:
// 65536 x 4096, bf16, an infinity in a token's last place, 1.07 ms for that token, 19.6 ms for 64 of them.
template <typename T>
__device__ __forceinline__ float product_in_order(const ProductArgs& a, uint64_t r, uint64_t t) {
    const uint8_t* row = a.msg + r * a.row_bytes;
    const T* x = static_cast<const T*>(a.in) + t * a.in_ld;
    const uint32_t per = a.block / 8;
    float sum = 0.f;
#pragma unroll 1
    for (uint64_t w = 0; 8 * w < a.cols; ++w) {
        const uint8_t* block = row + w / per * (4 + a.block / 2);
        const float unit = *reinterpret_cast<const float*>(block) * (16.f / 15.f);
        const uint32_t word = *reinterpret_cast<const uint32_t*>(block + 4 + 4 * (w % per));
        float part = 0.f;                                         // a code counts as (2 code - 15) / 16: no sum is infinite before y is
#pragma unroll 1
        for (int e = 0; e < 8; ++e)
            if (8 * w + e < a.cols) part = fmaf((float)(2 * (int)(word >> (4 * e) & 15u) - 15) * 0.0625f, (float)x[8 * w + e], part);
        sum = fmaf(unit, part, sum);
        if (sum != sum) break;                                    // and NaN stays
    }
    return sum;
}

template <typename T>
__device__ __forceinline__ void product_store(const ProductArgs& a, uint64_t r, uint64_t t, float v) {
    if (!(fabsf(v) < __builtin_huge_valf())) v = product_in_order<T>(a, r, t);
    static_cast<T*>(a.out)[t * a.out_ld + r] = (T)v;
}

// 128 columns of a lane's row: four words and the scales of the block they lie in (of the two blocks, where a block is 64 columns).
// Words 2 h and 2 h + 1 of all lanes j of the row go into matrix instruction h, which must not mix blocks: word t of lane j starts at
// column 32 j + 8 t, or at 64 floor(t / 2) + 16 j + 8 (t % 2) where a block is 64 columns.
template <bool NARROW>
struct Codes {
    uint32_t w[4];
    float scale[NARROW ? 2 : 1];
};
template <bool NARROW>
__device__ __forceinline__ uint32_t word_column(uint32_t t, uint32_t j) { return NARROW ? 64 * (t / 2) + 16 * j + 8 * (t % 2) : 32 * j + 8 * t; }

template <bool NARROW>
__device__ __forceinline__ void load_codes(Codes<NARROW>& c, const uint8_t* row, uint32_t block_log2, uint64_t col, uint32_t j) {
    if constexpr (NARROW) {
        const uint8_t* p = row + col / 64 * 36;
        c.scale[0] = *reinterpret_cast<const float*>(p);
        c.scale[1] = *reinterpret_cast<const float*>(p + 36);
        const u32x2 a = *reinterpret_cast<const u32x2_at4*>(p + 4 + 8 * j), b = *reinterpret_cast<const u32x2_at4*>(p + 40 + 8 * j);
        c.w[0] = a.x; c.w[1] = a.y; c.w[2] = b.x; c.w[3] = b.y;
    } else {
        const uint8_t* p = row + (col >> block_log2) * (4 + (1u << block_log2) / 2);
        c.scale[0] = *reinterpret_cast<const float*>(p);
        const u32x4 v = *reinterpret_cast<const u32x4_at4*>(p + 4 + (col & ((1u << block_log2) - 1)) / 2 + 16 * j);
        c.w[0] = v.x; c.w[1] = v.y; c.w[2] = v.z; c.w[3] = v.w;
    }
}
// The row's last columns, fewer than 128: words that are not there are 0, and nothing behind the row is read.
template <bool NARROW>
__device__ __forceinline__ void load_codes_tail(Codes<NARROW>& c, const uint8_t* row, uint32_t block_log2, uint64_t col, uint64_t cols, uint32_t j) {
#pragma unroll
    for (int b = 0; b < (NARROW ? 2 : 1); ++b) {
        const uint64_t at = col + 64 * b;
        c.scale[b] = at < cols ? *reinterpret_cast<const float*>(row + (at >> block_log2) * (4 + (1u << block_log2) / 2)) : 0.f;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint64_t at = col + word_column<NARROW>(t, j);
        c.w[t] = at < cols ? *reinterpret_cast<const uint32_t*>(row + (at >> block_log2) * (4 + (1u << block_log2) / 2) + 4 + (at & ((1u << block_log2) - 1)) / 2) : 0u;
    }
}

// 2^p, for p from -126 to 127.
__device__ __forceinline__ float power2_of(int p) { return __uint_as_float((uint32_t)(p + 127) << 23); }
// The largest p for which 2^p x is at most `limit`, just below 2^31, of an |x| with these bits: -98 to 149 (2^149 makes an integer of any x).  At -98, for |x| of
// 3.1e38 and more, 2^(kExponent - p) is infinite, and results are made in order.
__device__ __forceinline__ int power_of(uint32_t bits, float limit) {
    const int p = kExponent + 127 - (int)(bits >> 23), q = p > 149 ? 149 : p;
    return ldexpf(__uint_as_float(bits), q) > limit ? q - 1 : q;
}

// op over 8 or 16 adjacent lanes, in all of them: each lane with its mirror image, then with the others of its four.
template <int CTRL, typename V>
__device__ __forceinline__ V other_lane(V v) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LANES, typename V, typename F>
__device__ __forceinline__ V over_lanes(V v, F op) {
    if (LANES == 16) v = op(v, other_lane<0x140>(v));             // row_mirror
    v = op(v, other_lane<0x141>(v));                              // row_half_mirror
    v = op(v, other_lane<0x4E>(v));                               // quad_perm 2 3 0 1
    return op(v, other_lane<0xB1>(v));                            // quad_perm 1 0 3 2
}

// Eight columns of x, zero behind the last.
template <typename T>
struct EightOf {
    typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
template <typename T>
__device__ __forceinline__ typename EightOf<T>::Raw load_eight(const T* x, uint32_t col, uint32_t cols) {
    using Raw = typename EightOf<T>::Raw;
    if (col + 8 <= cols) return *reinterpret_cast<const Raw*>(x + col);
    Raw raw;
#pragma unroll
    for (int e = 0; e < 8; ++e) raw[e] = col + e < cols ? x[col + e] : (T)0.f;
    return raw;
}
// The bits of the largest of N magnitudes; NaN is above all.
template <int N>
__device__ __forceinline__ uint32_t largest_bits(const float (&v)[N]) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const uint32_t bits = __float_as_uint(v[e]) & 0x7FFFFFFFu;
        most = bits > most ? bits : most;
    }
    return most;
}

// Byte b of four words, as word b.
__device__ __forceinline__ void transpose_bytes(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t (&out)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w1, w0, 0x05010400u), b = __builtin_amdgcn_perm(w3, w2, 0x05010400u);
    const uint32_t c = __builtin_amdgcn_perm(w1, w0, 0x07030602u), d = __builtin_amdgcn_perm(w3, w2, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// Sixteen adjacent lanes, lane u with columns 8 u .. 8 u + 7 of a chunk (raw), write a token's part of the chunk's record.
template <typename T, int TT, bool NARROW>
__device__ void make_record(uint32_t tok, uint32_t u, typename EightOf<T>::Raw raw, uint8_t* record) {
    using R = Record<T, TT, NARROW>;
    constexpr int LANES = NARROW ? 8 : 16;                        // of a block
    const uint32_t t = NARROW ? u / 8 * 2 + u % 2 : u % 4, j = NARROW ? u % 8 / 2 : u / 4;
    if constexpr (sizeof(T) == 2) {
        R::x(record)[(4 * t + j) * R::rows + tok] = in_code_order(__builtin_bit_cast(u32x4, raw));
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += (float)raw[e];
        sum = over_lanes<LANES>(sum, [](float x, float y) { return x + y; });
        if (u % LANES == 0) static_cast<float*>(R::start(record))[u / LANES * R::rows + tok] = -kCentre * sum;
    } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = raw[e];
        // 2^power x, rounded, plus 128 in all digits but the highest: its bytes are the digits, their sign bits turned over where 128 was added
        const uint32_t most = over_lanes<LANES>(largest_bits(x), [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        const int power = power_of(most, kMostDigits);
        const bool finite = most < 0x7F800000u;                   // (if not, the block counts as NaN, whatever its digits are)
        uint32_t v[8], bytes[4][2];                               // of a digit: the odd columns apart from the even ones
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (uint32_t)(finite ? (int32_t)rintf(ldexpf(x[e], power)) : 0) + 0x808080u;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            uint32_t lowest_first[4];
            transpose_bytes(v[o], v[2 + o], v[4 + o], v[6 + o], lowest_first);
#pragma unroll
            for (int d = 0; d < 4; ++d) bytes[d][o] = lowest_first[3 - d] ^ (d ? 0x80808080u : 0u);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t at = (((t / 2) * 4 + j) * R::rows + 4 * tok + d) * 16 + 8 * (t % 2);
            *reinterpret_cast<u32x2*>(record + at) = u32x2{bytes[d][0], bytes[d][1]};
            constexpr int kOff = (int)0xF1F1F1F1;                 // -15 each
            int32_t sum = __builtin_amdgcn_sdot4((int)bytes[d][0], kOff, __builtin_amdgcn_sdot4((int)bytes[d][1], kOff, 0, false), false);
            sum = over_lanes<LANES>(sum, [](int32_t x, int32_t y) { return x + y; });
            if (u % LANES == 0) static_cast<int32_t*>(R::start(record))[u / LANES * R::rows + 4 * tok + d] = sum;
        }
        if (u % LANES == 0) R::unit(record)[u / LANES * (TT * 4) + tok] = finite ? power2_of(kExponent - power) : __builtin_nanf("");
    }
}

// The records, for all workgroups: 16 threads per chunk and token.
template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(256) product_records_kernel(ProductShape a, uint8_t* panel) {
    const uint64_t chunk = blockIdx.x;
    const uint32_t tok = threadIdx.x / 16 + 16 * blockIdx.y, u = threadIdx.x % 16;
    if (tok >= a.tokens) return;
    const T* x = static_cast<const T*>(a.in) + tok * a.in_ld;
    make_record<T, TT, NARROW>(tok, u, load_eight(x, (uint32_t)chunk * kChunk + 8 * u, (uint32_t)a.cols), panel + chunk * Record<T, TT, NARROW>::bytes);
}

// The products of a chunk of codes, 16 RT rows, with the chunk's record of x.
template <typename T, int TT, int RT, bool NARROW>
__device__ __forceinline__ void multiply(const Codes<NARROW> (&c)[RT], uint8_t* rec, uint32_t n, uint32_t j, CodeMasks masks,
                                         float (&sum)[RT][TT][4 / kTokenRows<T>]) {
    using R = Record<T, TT, NARROW>;
    constexpr bool kInteger = sizeof(T) == 4;
    constexpr int H = NARROW ? 2 : 1, PER = 4 / kTokenRows<T>, W = kInteger ? 2 : 4;       // blocks of a chunk; tokens of a lane; operands of a chunk
    using Operand = std::conditional_t<kInteger, i32x4, Eight<Coded<T>>>;
    using Sums = std::conditional_t<kInteger, i32x4, f32x4>;
    Operand codes[RT][W];
    float unit[RT][H];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if constexpr (kInteger)
                codes[r][w] = i32x4{(int)(c[r].w[2 * w] << 1 & 0x1E1E1E1Eu), (int)(c[r].w[2 * w] >> 3 & 0x1E1E1E1Eu),
                                    (int)(c[r].w[2 * w + 1] << 1 & 0x1E1E1E1Eu), (int)(c[r].w[2 * w + 1] >> 3 & 0x1E1E1E1Eu)};
            else codes[r][w] = code_operand<T>(c[r].w[w], masks);
        }
#pragma unroll
        for (int b = 0; b < H; ++b) unit[r][b] = c[r].scale[b] * (kInteger ? 1.f / 15.f : kPerCode);
    }
    struct Left {
        Operand x[W];
        Sums start[H];
        float count[H];
    };
    auto load = [&](Left& v, int t) {
#pragma unroll
        for (int w = 0; w < W; ++w) v.x[w] = __builtin_bit_cast(Operand, R::x(rec)[(4 * w + j) * R::rows + 16 * t + n]);
#pragma unroll
        for (int b = 0; b < H; ++b) {
            v.start[b] = *reinterpret_cast<const Sums*>(static_cast<uint32_t*>(R::start(rec)) + b * R::rows + 16 * t + 4 * j);
            if constexpr (kInteger) v.count[b] = R::unit(rec)[b * (TT * 4) + 4 * t + j];
        }
    };
    Left left[2];
    load(left[0], 0);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        if (t + 1 < TT) load(left[(t + 1) % 2], t + 1);
        const Left& v = left[t % 2];
#pragma unroll
        for (int b = 0; b < H; ++b)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                Sums p = v.start[b];
#pragma unroll
                for (int w = b * (W / H); w < (b + 1) * (W / H); ++w) {
                    if constexpr (kInteger) p = __builtin_amdgcn_mfma_i32_16x16x64_i8(v.x[w], codes[r][w], p, 0, 0, 0);
                    else p = matrix_fma(v.x[w], codes[r][w], p);
                }
                if constexpr (kInteger) {                         // the factors one after the other, smallest first: no product leaves fp32's range before y does
                    const float high = (float)((p[0] << 8) + p[1]), low = (float)((p[2] << 8) + p[3]);
                    const float w = fmaf(high, 0x1p-14f, low * 0x1p-30f);
                    sum[r][t][0] = fmaf(unit[r][b] * w, v.count[b], sum[r][t][0]);
                } else {
#pragma unroll
                    for (int i = 0; i < PER; ++i) sum[r][t][i] = fmaf(unit[r][b], p[i], sum[r][t][i]);
                }
            }
        if constexpr (TT > kFewTiles<T>) {                        // what is asked for, and left to do, beyond the next tile takes registers (32 x 65536 x 4096, bf16: 69 us)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < PER; ++i) asm volatile("" : "+v"(sum[r][t][i]));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// More tokens: a workgroup takes 256 rows, chunk after chunk, its waves 32 rows each against the same x in LDS.  61 x 16001 x 4099, bf16, in blocks of 64: 24.4 us,
// vector instructions 31 % of the clocks, matrix instructions 18 %; two waves on a SIMD wait for one another at every chunk.
template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(kThreads) product_kernel(ProductShape a) {
    constexpr int RT = kRowTiles;
    using R = Record<T, TT, NARROW>;
    constexpr int PER = 4 / kTokenRows<T>;                        // tokens of a lane and matrix instruction
    constexpr uint32_t record = R::bytes, kAll = record / 16, kPieces = (kAll + kThreads - 1) / kThreads;      // x of a chunk, in 16-byte pieces; of a thread
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t tokens = (uint32_t)a.tokens;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane & 15, j = lane >> 4;
    const uint64_t c0 = (uint64_t)blockIdx.y * a.plan.part_chunks, all_chunks = (a.cols + kChunk - 1) / kChunk;
    const uint32_t chunks = (uint32_t)(all_chunks - c0 < a.plan.part_chunks ? all_chunks - c0 : a.plan.part_chunks);
    const uint32_t block_log2 = 31 - __builtin_clz(a.block);

    const uint64_t first = a.row0 + ((uint64_t)blockIdx.x * kWaves + wave) * (16 * RT);
    const uint8_t* row[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {                                // rows behind the last read the last one, and are not stored
        const uint64_t at = first + 16 * r + n;
        row[r] = a.msg + (at < a.rows ? at : a.rows - 1) * a.row_bytes;
    }
    float sum[RT][TT][PER];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < PER; ++i) sum[r][t][i] = 0.f;

    // x goes through LDS, a chunk ahead by way of registers, and codes are on their way two chunks ahead.  (Behind the end the last ones are read again: no
    // branch, so that loads can be counted.)
    const uint32_t whole = chunks - (c0 + chunks == all_chunks && a.cols % kChunk ? 1 : 0);    // without the ragged end
    const u32x4* x_from = reinterpret_cast<const u32x4*>(a.panel + c0 * record);
    auto bring = [&](u32x4 (&v)[kPieces], uint32_t c) {
        const u32x4* from = x_from + (uint64_t)(c < chunks ? c : chunks - 1) * kAll;
#pragma unroll
        for (uint32_t q = 0; q < kPieces; ++q) v[q] = from[q * kThreads + threadIdx.x < kAll ? q * kThreads + threadIdx.x : kAll - 1];
    };
    auto put = [&](const u32x4 (&v)[kPieces], uint32_t c) {
#pragma unroll
        for (uint32_t q = 0; q < kPieces; ++q)
            if (q * kThreads + threadIdx.x < kAll) reinterpret_cast<u32x4*>(lds + (c & 1) * record)[q * kThreads + threadIdx.x] = v[q];
    };
    const CodeMasks masks = code_masks<Coded<T>>();
    auto use = [&](const Codes<NARROW> (&codes)[RT], uint32_t c) { multiply<T, TT, RT, NARROW>(codes, lds + (c & 1) * record, n, j, masks, sum); };
    u32x4 x[kPieces];
    bring(x, 0);
    if (whole) {
        Codes<NARROW> ring[2][RT];
        auto fetch = [&](Codes<NARROW> (&codes)[RT], uint32_t c) {
            const uint64_t col = (c0 + (c < whole ? c : whole - 1)) * kChunk;
#pragma unroll
            for (int r = 0; r < RT; ++r) load_codes<NARROW>(codes[r], row[r], block_log2, col, j);
        };
        fetch(ring[0], 0);
        fetch(ring[1], 1);
        put(x, 0);
        __syncthreads();
        for (uint32_t c = 0; c < whole; c += 2) {
#pragma unroll
            for (uint32_t o = 0; o < 2; ++o) {
                if (c + o >= whole) break;
                bring(x, c + o + 1);
                use(ring[o], c + o);
                fetch(ring[o], c + o + 2);
                put(x, c + o + 1);
                __syncthreads();
            }
        }
    } else {
        put(x, 0);
        __syncthreads();
    }
    if (whole < chunks) {
        Codes<NARROW> codes[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) load_codes_tail<NARROW>(codes[r], row[r], block_log2, (c0 + whole) * kChunk, a.cols, j);
        use(codes, whole);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint64_t at = first + 16 * r + n;
                const uint32_t tok = (4 * t + j) * PER + i;
                if (at >= a.rows || tok >= tokens) continue;
                if (a.partial) a.partial[((uint64_t)blockIdx.y * tokens + tok) * a.rows + at] = sum[r][t][i];
                else product_store<T>(a, at, tok, sum[r][t][i]);
            }
}

// Few tokens: codes go through LDS, too, 128 rows of 256 columns at a time, so that memory is read in rows of 128 bytes and more (see product_one_kernel) and a
// compute unit has as much under way as it multiplies.  While a stage is multiplied the next one's loads are on their way into registers; then it goes into
// the other half of the LDS.  A row's part of a stage is read as it lies in the message, in nine pieces of 16 bytes, scales among the codes: a load that
// gathers scales alone costs the memory pipeline as much as one that brings 16 bytes a lane (2 x 65536 x 4096, blocks of 256, 30.7 us; with scales read
// apart a quarter more).  Blocks of more than 256 columns are read in eight pieces, and their scales once a block (of 2048: 31.0 us).
//   2 tokens of 65536 x 4096 read 4.6 TB/s, 16 tokens 3.6.  16 x 4096 x 16384, fp16: 14.4 us, 2.5 TB/s: 190 vector instructions of a wave and stage, 46 % of the
// clocks, and four stages of each workgroup, of which the first one's reads have nothing beside them.
// Slower, when x was held in digits: two stages ahead (registers; 22.8 us for 19.4), workgroups of 256 rows (2 x 65536 x 4096 46.8 for 42.9).
constexpr uint32_t kStageChunks = 2, kStageCols = kStageChunks * kChunk;                   // of a stage
static_assert(kStageCols == kStageColumns);

template <typename T, int TT, bool NARROW>
struct Stage {
    static constexpr uint32_t rows = 16 * kWaves, codes = rows * kRowPieces * 16, scales = rows * 4;
    static constexpr uint32_t bytes = codes + scales + kStageChunks * Record<T, TT, NARROW>::bytes;
};

template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(kThreads) product_tiles_kernel(ProductShape a) {
    using S = Stage<T, TT, NARROW>;
    static_assert(16 * kStageChunks * TT * kTileTokens<T> <= kThreads, "a thread has eight columns of x");
    using R = Record<T, TT, NARROW>;
    using Raw = typename EightOf<T>::Raw;
    constexpr int PER = 4 / kTokenRows<T>;
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t tokens = (uint32_t)a.tokens;
    constexpr uint32_t record = R::bytes, half = S::bytes;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane & 15, j = lane >> 4;
    const uint32_t block_log2 = 31 - __builtin_clz(a.block), pitch = 4 + a.block / 2;
    const uint64_t all_stages = (a.cols + kStageCols - 1) / kStageCols;
    const uint32_t cols = (uint32_t)a.cols, s0 = blockIdx.y * a.plan.part_chunks;          // (of stages here)
    const uint32_t stages = (uint32_t)(all_stages - s0 < a.plan.part_chunks ? all_stages - s0 : a.plan.part_chunks);
    const uint64_t first = a.row0 + (uint64_t)blockIdx.x * S::rows;

    // what the thread brings: two pieces of codes (some a third), a long block's scale, and x
    const bool apart = scales_apart(block_log2);
    const uint32_t row_pieces = stage_pieces(block_log2), row_bytes = (uint32_t)a.row_bytes;    // (below 2^28)
    auto row_at = [&](uint32_t r) { return a.msg + (first + r < a.rows ? first + r : a.rows - 1) * a.row_bytes; };
    constexpr uint32_t PIECES = (S::rows * kRowPieces + kThreads - 1) / kThreads;
    const uint8_t* from[PIECES];
    uint32_t piece_at[PIECES], piece_to[PIECES];
#pragma unroll
    for (uint32_t i = 0; i < PIECES; ++i) {
        const uint32_t q = i * kThreads + threadIdx.x, in = apart ? q / (kRowPieces - 1) : q / kRowPieces, r = in < S::rows ? in : S::rows - 1;
        from[i] = row_at(r);
        piece_at[i] = (q - in * row_pieces) * 16;
        piece_to[i] = r * kRowPieces * 16 + piece_at[i];
    }
    const bool has_third = (PIECES - 1) * kThreads + threadIdx.x < S::rows * row_pieces, has_scale = apart && threadIdx.x < S::rows;
    const uint8_t* scale_row = row_at(threadIdx.x % S::rows);
    const bool has_end = first + S::rows >= a.rows;               // of the message
    const uint32_t x_tok = threadIdx.x / (16 * kStageChunks), x_unit = threadIdx.x % (16 * kStageChunks);
    const T* x_row = static_cast<const T*>(a.in) + (x_tok < tokens ? x_tok : tokens - 1) * a.in_ld;
    struct Brought {
        u32x4 codes[PIECES];
        float scale;
        Raw x;
        uint32_t back;                                            // words that a piece which would end behind the message was read too early by
    };
    auto bring = [&](Brought& v, uint32_t s) {
        const uint32_t col = (s0 + s) * kStageCols, in_block = col & (a.block - 1), block_at = stage_scale(col, block_log2), at = stage_codes(col, block_log2);
        v.back = 0;
        if (col + kStageCols <= cols) {                           // all blocks are there, and a last piece may end in the next row ...
            if (has_end && at + row_pieces * 16 > row_bytes) {    // ... if there is one
                v.back = words_back(at, row_pieces, row_bytes);
#pragma unroll
                for (uint32_t i = 0; i < PIECES; ++i) {
                    if (i + 1 < PIECES || has_third) v.codes[i] = *reinterpret_cast<const u32x4_at4*>(from[i] + piece_read(at + piece_at[i], row_bytes));
                }
            } else {
#pragma unroll
                for (uint32_t i = 0; i < PIECES; ++i)
                    if (i + 1 < PIECES || has_third) v.codes[i] = *reinterpret_cast<const u32x4_at4*>(from[i] + (at + piece_at[i]));
            }
            v.x = *reinterpret_cast<const Raw*>(x_row + (col + 8 * x_unit));
        } else {                                                  // words that are not there are 0
#pragma unroll
            for (uint32_t i = 0; i < PIECES; ++i)
                if (i + 1 < PIECES || has_third)
#pragma unroll
                    for (uint32_t w = 0; w < 4; ++w) {
                        const uint32_t word = at + piece_at[i] + 4 * w;
                        v.codes[i][w] = word < row_bytes ? *reinterpret_cast<const uint32_t*>(from[i] + word) : 0u;
                    }
            v.x = load_eight(x_row, col + 8 * x_unit, cols);
        }
        if (has_scale && (in_block == 0 || s == 0)) v.scale = *reinterpret_cast<const float*>(scale_row + block_at);
    };
    auto put = [&](Brought& v, uint8_t* to) {
        if (v.back)
#pragma unroll
            for (uint32_t i = 0; i < PIECES; ++i)
                if (piece_at[i] == (kRowPieces - 1) * 16) {
                    const Front front = moved_to_front(v.back, v.codes[i].y, v.codes[i].z, v.codes[i].w);
                    v.codes[i].x = front.x;
                    v.codes[i].y = front.y;
                }
#pragma unroll
        for (uint32_t i = 0; i < PIECES; ++i)
            if (i + 1 < PIECES || has_third) *reinterpret_cast<u32x4*>(to + piece_to[i]) = v.codes[i];
        if (has_scale) reinterpret_cast<float*>(to + S::codes)[threadIdx.x] = v.scale;
        uint8_t* records = to + S::codes + S::scales;
        if (x_tok < tokens) make_record<T, TT, NARROW>(x_tok, x_unit % 16, v.x, records + x_unit / 16 * record);
    };

    float sum[1][TT][PER];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int i = 0; i < PER; ++i) sum[0][t][i] = 0.f;
    const uint32_t my_row = wave * 16 + n;
    // of the lane's row in a half: chunk c's scale and codes; with blocks of 64 block b's are 36 b from the first
    const uint32_t block = my_row * kRowPieces * 16, scale_at = apart ? S::codes + 4 * my_row : block, scale_step = a.block == kChunk ? pitch : 0;
    const uint32_t codes_at = block + (apart ? 0 : 4) + 16 * j, codes_step = a.block == kChunk ? pitch : kChunk / 2;
    const CodeMasks masks = code_masks<Coded<T>>();
    auto use = [&](uint8_t* half_at) {
#pragma unroll
        for (uint32_t c = 0; c < kStageChunks; ++c) {
            Codes<NARROW> codes[1];
            if constexpr (NARROW) {
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    const uint8_t* p = half_at + block + (2 * c + h) * 36;
                    codes[0].scale[h] = *reinterpret_cast<const float*>(p);
                    const u32x2 v = *reinterpret_cast<const u32x2_at4*>(p + 4 + 8 * j);
                    codes[0].w[2 * h] = v.x;
                    codes[0].w[2 * h + 1] = v.y;
                }
            } else {
                codes[0].scale[0] = *reinterpret_cast<const float*>(half_at + scale_at + c * scale_step);
                const u32x4 v = *reinterpret_cast<const u32x4_at4*>(half_at + codes_at + c * codes_step);
#pragma unroll
                for (int w = 0; w < 4; ++w) codes[0].w[w] = v[w];
            }
            multiply<T, TT, 1, NARROW>(codes, half_at + S::codes + S::scales + c * record, n, j, masks, sum);
        }
    };
    // Stage s is multiplied out of one half of the LDS while stage s + 1 is on its way.  (The last one again behind the end: no branch.)
    Brought coming;
    bring(coming, 0);
    put(coming, lds);
    __syncthreads();
    for (uint32_t s = 0; s < stages; ++s) {
        bring(coming, s + 1 < stages ? s + 1 : s);
        use(lds + (s & 1) * half);
        put(coming, lds + ((s + 1) & 1) * half);
        __syncthreads();
    }
    const uint64_t at = first + my_row;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t tok = (4 * t + j) * PER + i;
            if (at >= a.rows || tok >= tokens) continue;
            if (a.partial) a.partial[((uint64_t)blockIdx.y * tokens + tok) * a.rows + at] = sum[0][t][i];
            else product_store<T>(a, at, tok, sum[0][t][i]);
        }
}

// One token: rows of codes are read whole, which costs the memory pipeline a third of what sixteen rows of 64 bytes cost a load, and meet x in
// registers.  A lane keeps 32 columns of x for all the rows of its wave, G lanes hold a row, and a load takes 64 / G rows of 32 G columns.
//   16-bit types: a matrix instruction of 4 x 4 blocks, lane l's operands row and column l % 4 of block l / 4, of which the lane's own product stands on the
// diagonal, in its register l % 4; the other twelve sums are of no use and cost nothing that is short.
//   fp32: x is written in eight signed digits of four bits, 16^d apart, with an exponent per 32 columns: eight codes (less 8, so that they are signed) meet
// eight digits in one instruction.
// The lanes of a row are joined by a tree of lane shifts.  65536 x 4096, bf16: 24.9 us, 5.7 TB/s, the
// vector units busy 70 % of the time, the matrix units 16 %; fp32 31 us.
constexpr uint32_t kLaneCols = 32;
constexpr int kNibbles = 8;
constexpr float kMostNibbles = 2004317952.f;                      // 7 (16^7 + .. + 16 + 1), as a number of fp32

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float add_shifted(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROW_MASK, 0xF, false));
}
// The sum over G adjacent lanes, in the last of them.
template <int G>
__device__ __forceinline__ float lanes_total(float v) {
    v = add_shifted<0x111, 0xF>(v);
    v = add_shifted<0x112, 0xF>(v);
    if constexpr (G >= 16) {
        v = add_shifted<0x114, 0xF>(v);
        v = add_shifted<0x118, 0xF>(v);
    }
    if constexpr (G >= 32) v = add_shifted<0x142, 0xA>(v);
    if constexpr (G >= 64) v = add_shifted<0x143, 0xC>(v);
    return v;
}

// What a lane has of x, in one of two forms.
template <typename T>
struct Own {                                                      // 16-bit types: words in the order of codes, and what a product starts from
    u32x4 x[4];
    float start;
    CodeMasks masks;

    // `missing` of the words that come before the lane's are read with it, and count for nothing.
    __device__ void read(const T* x_of, uint64_t col, uint64_t cols) {
        using Raw = typename EightOf<T>::Raw;
        const uint32_t missing = missing_words(col, cols);
        float sum = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < 4; ++w) {
            Raw raw;
            if (col + kLaneCols <= cols) {
                raw = *reinterpret_cast<const Raw*>(x_of + col + 8 * w);
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) {
                    const uint64_t c = col + 8 * w + e - 8 * missing;
                    raw[e] = w >= missing && c < cols ? x_of[c] : (T)0.f;
                }
            }
            x[w] = in_code_order(__builtin_bit_cast(u32x4, raw));
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (float)raw[e];
        }
        start = -kCentre * sum;
        masks = code_masks<T>();
    }
    __device__ float product(u32x4 words, float scale) const {
        f32x4 p = {start, start, start, start};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const u32x4 codes = __builtin_bit_cast(u32x4, code_operand<T>(words[w], masks));
            p = own_products<T>(codes.xy, x[w].xy, p);
            p = own_products<T>(codes.zw, x[w].zw, p);
        }
        const uint32_t lane = threadIdx.x;
        const float even = lane & 2 ? p.z : p.x, odd = lane & 2 ? p.w : p.y;
        return scale * kPerCode * (lane & 1 ? odd : even);
    }
};
template <>
struct Own<float> {                                               // digits; sum v as high and low halves of v; what v counts, over 2^kExponent
    i32x4 digits[kNibbles];
    int32_t high, low;
    float count;

    __device__ float product(u32x4 words, float scale) const {
        int32_t dot[kNibbles];
#pragma unroll
        for (int d = 0; d < kNibbles; ++d) dot[d] = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int d = 0; d < kNibbles; ++d) dot[d] = __builtin_amdgcn_sdot8((int32_t)(words[w] ^ 0x88888888u), digits[d][w], dot[d], false);   // code - 8
        // sum (2 code - 15) v = 2 sum (code - 8) v + sum v
        const int32_t upper = ((dot[7] * 16 + dot[6]) * 16 + dot[5]) * 16 + dot[4], lower = ((dot[3] * 16 + dot[2]) * 16 + dot[1]) * 16 + dot[0];
        const float v = fmaf((float)(2 * upper + high), 0x1p-14f, (float)(2 * lower + low) * 0x1p-30f);
        return scale * (1.f / 15.f) * v * count;                  // (one after the other: see multiply)
    }
};

template <typename T, int G>
__global__ void __launch_bounds__(kThreads) product_one_kernel(ProductShape a) {
    constexpr int AT_ONCE = 64 / G, AHEAD = 4;                    // rows of a load, loads under way
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / G, l = lane % G;
    const uint32_t row_waves = a.plan.row_waves, col_waves = kWaves / row_waves, rw = wave % row_waves, cw = wave / row_waves;
    const uint32_t wave_rows = a.plan.wave_rows, rows_here = row_waves * wave_rows, loads = wave_rows / AT_ONCE;
    const uint64_t first = a.row0 + (uint64_t)blockIdx.x * rows_here;
    const uint32_t block_log2 = 31 - __builtin_clz(a.block);
    const uint32_t lanes = col_waves * G;                         // lanes that hold different columns
    float* totals = reinterpret_cast<float*>(lds);                // [column wave][row of the workgroup]
    float* mine = totals + cw * rows_here + rw * wave_rows;
    const T* x = static_cast<const T*>(a.in);
    for (uint64_t slice = 0; slice < a.cols; slice += lanes * kLaneCols) {
        const uint64_t col = slice + (cw * G + l) * kLaneCols;
        const bool some = col < a.cols;                           // (if not, the lane counts for nothing)
        const LaneRead read = lane_read(col, a.cols, block_log2);
        struct Load {
            u32x4 w;
            float scale;
        };
        auto fetch = [&](Load& v, uint32_t q) {                   // the q-th rows, or again the last: no branch, so that loads can be counted
            const uint64_t at = first + rw * wave_rows + (q < loads ? q : loads - 1) * AT_ONCE + g, row = at < a.rows ? at : a.rows - 1;
            const uint8_t* p = a.msg + row * a.row_bytes;
            v.scale = *reinterpret_cast<const float*>(p + read.scale);
            v.w = *reinterpret_cast<const u32x4_at4*>(p + read.codes);
        };
        Load ring[AHEAD];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) fetch(ring[s], s);
        Own<T> own;
        if constexpr (sizeof(T) == 2) {
            own.read(x, col, a.cols);
        } else {
            // the workgroup writes this stretch of x in digits, [digit][lane]: a thread takes eight columns, four threads a lane's 32
            i32x4* digits = reinterpret_cast<i32x4*>(totals + kWaves * wave_rows);
            int32_t* highs = reinterpret_cast<int32_t*>(digits + kNibbles * lanes);
            int32_t* lows = highs + lanes;
            float* counts = reinterpret_cast<float*>(lows + lanes);
            if (slice) __syncthreads();
            for (uint32_t w = threadIdx.x; w < lanes * 4; w += kThreads) {
                const uint64_t at = slice + 8 * w;
                float v[8];
                if (at + 8 <= a.cols) {
                    const EightOf<float>::Raw raw = *reinterpret_cast<const EightOf<float>::Raw*>(x + at);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = raw[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = at + e < a.cols ? (float)x[at + e] : 0.f;
                }
                uint32_t most = largest_bits(v);
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    const uint32_t other = (uint32_t)__shfl_xor((int)most, o);
                    most = other > most ? other : most;
                }
                const int power = power_of(most, kMostNibbles);
                const bool finite = most < 0x7F800000u;
                // 2^power x, rounded, plus 8 in all digits: its digits of four bits are the signed ones plus 8, whose highest bits are turned over
                uint32_t out[kNibbles], nibbles[8];
                int32_t high = 0, low = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t rounded = finite ? (int32_t)rintf(ldexpf(v[e], power)) : 0;
                    high += rounded >> 16;
                    low += rounded & 0xFFFF;
                    nibbles[e] = ((uint32_t)rounded + 0x88888888u) ^ 0x88888888u;
                }
                // digit d of column e to place e of word d, the lowest digit first
#pragma unroll
                for (int odd = 0; odd < 2; ++odd) {
                    uint32_t pair[4], word[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        pair[p] = odd ? (nibbles[2 * p] >> 4 & 0x0F0F0F0Fu) | (nibbles[2 * p + 1] & 0xF0F0F0F0u)
                                      : (nibbles[2 * p] & 0x0F0F0F0Fu) | (nibbles[2 * p + 1] << 4 & 0xF0F0F0F0u);
                    transpose_bytes(pair[0], pair[1], pair[2], pair[3], word);
#pragma unroll
                    for (int b = 0; b < 4; ++b) out[2 * b + odd] = word[b];
                }
                const uint32_t place = (w % 4 + missing_words(slice + w / 4 * kLaneCols, a.cols)) % 4;
#pragma unroll
                for (int d = 0; d < kNibbles; ++d) reinterpret_cast<uint32_t*>(digits + d * lanes + w / 4)[place] = out[d];
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    high += __shfl_xor(high, o);
                    low += __shfl_xor(low, o);
                }
                if (w % 4 == 0) {
                    highs[w / 4] = high;
                    lows[w / 4] = low;
                    counts[w / 4] = finite ? power2_of(kExponent - power) : __builtin_nanf("");
                }
            }
            __syncthreads();
            const uint32_t from = cw * G + l;
#pragma unroll
            for (int d = 0; d < kNibbles; ++d) own.digits[d] = digits[d * lanes + from];
            own.high = highs[from];
            own.low = lows[from];
            own.count = counts[from];
        }
        auto use = [&](const Load& v, uint32_t q) {
            const float sum = lanes_total<G>(own.product(v.w, some ? v.scale : 0.f));
            if (l == G - 1) {
                float* to = mine + q * AT_ONCE + g;
                *to = slice ? *to + sum : sum;
            }
        };
        for (uint32_t q = 0; q < loads; q += AHEAD) {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                if (q + s >= loads) break;
                const Load now = ring[s];
                fetch(ring[s], q + s + AHEAD);
                use(now, q + s);
            }
        }
    }
    __syncthreads();
    for (uint32_t q = threadIdx.x; q < rows_here; q += kThreads) {
        const uint64_t at = first + q;
        if (at >= a.rows) break;
        float v = totals[q];
        for (uint32_t c = 1; c < col_waves; ++c) v += totals[c * rows_here + q];
        product_store<T>(a, at, 0, v);
    }
}

// Adds the parts.  A thread per row and token.
template <typename T>
__global__ void __launch_bounds__(256) product_join_kernel(ProductShape a) {
    const uint64_t r = a.row0 + (uint64_t)blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
    if (r >= a.rows) return;
    const float* from = a.partial + t * a.rows + r;
    const uint64_t step = a.tokens * a.rows;
    float v = 0.f;
    for (uint32_t p = 0; p < a.plan.parts; p += 4) {
        float w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = p + q < a.plan.parts ? from[(p + q) * step] : 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) v += w[q];
    }
    product_store<T>(a, r, t, v);
}

template <typename T>
int product_tiles(uint64_t tokens) {
    int tiles = 1;
    while ((uint64_t)tiles * kTileTokens<T> < tokens) tiles *= 2;
    return tiles;
}

// f(std::integral_constant<int, tiles>(), std::bool_constant<narrow>())
template <typename T, typename F>
void by_tiles(int tiles, bool narrow, F f) {
    auto with = [&](auto t) {
        if (narrow) f(t, std::true_type());
        else f(t, std::false_type());
    };
    if (tiles == 1) with(std::integral_constant<int, 1>());
    else if (tiles == 2) with(std::integral_constant<int, 2>());
    else if constexpr (kMostTiles<T> == 4) with(std::integral_constant<int, 4>());
    else if (tiles == 4) with(std::integral_constant<int, 4>());
    else with(std::integral_constant<int, 8>());
}

template <typename T>
uint32_t record_bytes(uint64_t tokens, bool narrow) {
    uint32_t bytes = 0;
    by_tiles<T>(product_tiles<T>(tokens), narrow, [&](auto t, auto n) { bytes = Record<T, decltype(t)::value, decltype(n)::value>::bytes; });
    return bytes;
}

// How many workgroups split the columns, where there are so many side by side and `most` could: until there are `want`, 32 at most.
uint32_t split(uint64_t want, uint64_t groups, uint64_t most) {
    uint64_t parts = want / groups;
    if (parts > most) parts = most;
    return parts < 1 ? 1 : parts > 32 ? 32 : (uint32_t)parts;
}

template <typename T>
ProductPlan product_plan(uint64_t rows, uint64_t cols, uint64_t tokens) {
    ProductPlan p{};
    const int tiles = product_tiles<T>(tokens);
    const uint64_t chunks = (cols + kChunk - 1) / kChunk;
    if (tiles <= kFewTiles<T>) {
        // Two workgroups for every compute unit where each has four stages, otherwise one where it has any: 4 x 16384 x 4096, fp32, 2 parts (256 workgroups)
        // 18.6 us, 4: 17.3, 6: 19.0; 16 x 20000 x 4096, bf16, blocks of 64, 1 part (157) 20.9, 2: 23.5, 3: 21.3; 16 x 4096 x 4096 4 parts (128) 13.1, 8 (of two
        // stages) 9.3, 16: 10.7; 16 x 5000 x 4096 6 parts (240) 10.6, 12: 12.0; 8 x 2048 x 2048 1 part 10.4, 8 (128 workgroups, a stage each): 7.0.
        const uint64_t stages = (chunks + kStageChunks - 1) / kStageChunks, groups = (rows + 16 * kWaves - 1) / (16 * kWaves);
        p.parts = split(512, groups, stages);
        if (stages < 4 * p.parts) p.parts = split(256, groups, stages);
        if (stages < 6) p.parts = 1;                              // (a stage takes 1.2 us where there are few workgroups, the launch that joins 2.6)
        p.part_chunks = (uint32_t)((stages + p.parts - 1) / p.parts);
        p.parts = (uint32_t)((stages + p.part_chunks - 1) / p.part_chunks);
        return p;
    }
    const uint64_t height = 16 * kRowTiles * kWaves, groups = (rows + height - 1) / height;
    // Workgroups split the columns until all compute units have one, and not one more, which would take as long again or add to what is joined: 61 x 16001 x
    // 4099, bf16, 3 parts 34.6 us, 4 (252 workgroups) 31.8, 8: 41.9; 64 x 65536 x 1024 1 part (256) 21.3, 2: 39.7; 64 x 2048 x 2048, fp32, 4 parts (of four
    // chunks) 17.2, 16 (128 workgroups, a chunk each) 11.0; 30 x 300 x 1000, bf16, 2 parts 16.8, 8: 10.5.
    p.parts = chunks < 4 ? 1 : split(256, groups, chunks);        // (a chunk takes 1.5 us where there are few workgroups, the launch that joins 2.6)
    p.part_chunks = (uint32_t)((chunks + p.parts - 1) / p.parts);
    p.parts = (uint32_t)((chunks + p.part_chunks - 1) / p.part_chunks);
    return p;
}

// product_one_kernel's calls: a row has four words.
bool by_rows(uint64_t tokens, uint64_t cols) { return tokens == 1 && cols > 24; }

// Scratch: the panel (of product_kernel), then the partial sums.
template <typename T>
uint64_t panel_bytes(uint64_t cols, uint64_t tokens, bool narrow) {
    return product_tiles<T>(tokens) > kFewTiles<T> ? (cols + kChunk - 1) / kChunk * record_bytes<T>(tokens, narrow) : 0;
}
template <typename T>
uint64_t scratch_bytes(uint64_t rows, uint64_t cols, uint64_t tokens, bool narrow) {
    if (by_rows(tokens, cols)) return 0;
    const ProductPlan plan = product_plan<T>(rows, cols, tokens);
    return panel_bytes<T>(cols, tokens, narrow) + (plan.parts > 1 ? plan.parts * tokens * rows * sizeof(float) : 0);
}

// Launches with as many workgroups as a launch takes: launch(first row, workgroups).
template <typename F>
void over_rows(uint64_t rows, uint64_t height, F launch) {
    const uint64_t groups = (rows + height - 1) / height;
    for (uint64_t g = 0; g < groups; g += kGroupsOfLaunch) launch(g * height, (unsigned)(groups - g < kGroupsOfLaunch ? groups - g : kGroupsOfLaunch));
}

template <typename T, int TT, bool NARROW>
void launch_product_tiles(ProductShape a, hipStream_t stream) {
    using S = Stage<T, TT, NARROW>;
    constexpr uint32_t lds = 2 * S::bytes;
    static_assert(lds <= 64 * 1024, "what a launch may ask for");
    over_rows(a.rows, S::rows, [&](uint64_t row0, unsigned groups) {
        a.row0 = row0;
        hipLaunchKernelGGL((product_tiles_kernel<T, TT, NARROW>), dim3(groups, a.plan.parts), dim3(kThreads), lds, stream, a);
    });
}

template <typename T, int TT, bool NARROW>
void launch_product_kernels(ProductShape a, hipStream_t stream) {
    if constexpr (TT <= kFewTiles<T>) {
        launch_product_tiles<T, TT, NARROW>(a, stream);
    } else {
        constexpr uint32_t lds = 2 * Record<T, TT, NARROW>::bytes;
        static_assert(lds <= 64 * 1024, "what a launch may ask for");
        hipLaunchKernelGGL((product_records_kernel<T, TT, NARROW>), dim3((unsigned)((a.cols + kChunk - 1) / kChunk), (unsigned)(a.tokens + 15) / 16), dim3(256), 0, stream, a,
                           static_cast<uint8_t*>(a.work));
        a.panel = static_cast<const uint8_t*>(a.work);
        over_rows(a.rows, 16 * kRowTiles * kWaves, [&](uint64_t row0, unsigned groups) {
            a.row0 = row0;
            hipLaunchKernelGGL((product_kernel<T, TT, NARROW>), dim3(groups, a.plan.parts), dim3(kThreads), lds, stream, a);
        });
    }
}

template <typename T, int G>
void launch_product_one(ProductShape a, hipStream_t stream) {
    constexpr uint32_t AT_ONCE = 64 / G;
    const uint64_t slices = (a.cols + G * kLaneCols - 1) / (G * kLaneCols);
    uint32_t col_waves = 1;
    while (col_waves < kWaves && col_waves < slices) col_waves *= 2;
    a.plan.row_waves = kWaves / col_waves;
    // Rows enough to be worth laying x out for, as long as there is a workgroup for every compute unit: 65536 x 4096, bf16, 8 rows a wave 31.6 us,
    // 16: 28.4, 32: 29.1, 64: 29.4; fp32 8: 38.0, 16: 32.8, 32: 31.5, 64: 33.6; 4096 x 16384, fp16, 8: 10.3 (512 workgroups), 16: 10.0, 32: 14.2 (128);
    // fp32 8: 15.8, 16: 14.1, 32: 18.8; 2048 x 2048, fp32, 1: 4.2, 4: 5.2, 16: 9.7.
    const uint64_t each = a.rows / (256ull * a.plan.row_waves) / AT_ONCE * AT_ONCE;
    a.plan.wave_rows = (uint32_t)(each < AT_ONCE ? AT_ONCE : each > 32 ? 32 : each);
    const uint64_t rows_here = (uint64_t)a.plan.row_waves * a.plan.wave_rows;
    const uint32_t bytes = kWaves * a.plan.wave_rows * 4 + (sizeof(T) == 4 ? col_waves * G * (kNibbles * 16 + 12) : 0);
    if (bytes > 64 * 1024)                                        // (fp32 and more than 8192 columns: 70 KB of digits; without it a launch may ask for 64 KB)
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(product_one_kernel<T, G>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    over_rows(a.rows, rows_here, [&](uint64_t row0, unsigned groups) {
        a.row0 = row0;
        hipLaunchKernelGGL((product_one_kernel<T, G>), dim3(groups), dim3(kThreads), bytes, stream, a);
    });
}

template <typename T>
void launch_product_of(const ProductArgs& args, hipStream_t stream) {
    const bool narrow = args.block == 64;
    for (uint64_t t0 = 0; t0 < args.tokens; t0 += kTokens<T>) {
        ProductShape a{};
        static_cast<ProductArgs&>(a) = args;
        a.tokens = args.tokens - t0 < kTokens<T> ? args.tokens - t0 : kTokens<T>;
        a.in = static_cast<const T*>(args.in) + t0 * args.in_ld;
        a.out = static_cast<T*>(args.out) + t0 * args.out_ld;
        if (by_rows(a.tokens, a.cols)) {
            if (a.cols <= 4 * kLaneCols) launch_product_one<T, 4>(a, stream);
            else if (a.cols <= 16 * kLaneCols) launch_product_one<T, 16>(a, stream);
            else if (a.cols <= 32 * kLaneCols) launch_product_one<T, 32>(a, stream);
            else launch_product_one<T, 64>(a, stream);
            continue;
        }
        a.plan = product_plan<T>(a.rows, a.cols, a.tokens);
        if (a.plan.parts > 1) a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(a.work) + panel_bytes<T>(a.cols, a.tokens, narrow));
        by_tiles<T>(product_tiles<T>(a.tokens), narrow, [&](auto t, auto n) { launch_product_kernels<T, decltype(t)::value, decltype(n)::value>(a, stream); });
        if (!a.partial) continue;
        over_rows(a.rows, 256, [&](uint64_t row0, unsigned groups) {
            a.row0 = row0;
            hipLaunchKernelGGL(product_join_kernel<T>, dim3(groups, (unsigned)a.tokens), dim3(256), 0, stream, a);
        });
    }
}

}  // namespace

uint64_t product_work_bytes(const ds_matrix& m) {
    uint64_t bytes = 0;
    by_dtype(m.dtype, [&](auto kind) {
        using T = decltype(kind);
        auto most = [&](uint64_t tokens) {                        // of the launches: whole ones and the last
            const uint64_t here = scratch_bytes<T>(m.rows, m.cols, tokens, m.block == 64);
            if (here > bytes) bytes = here;
        };
        if (m.tokens >= kTokens<T>) most(kTokens<T>);
        if (m.tokens % kTokens<T>) most(m.tokens % kTokens<T>);
    });
    return bytes;
}

hipError_t launch_product(const ProductArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_product_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
