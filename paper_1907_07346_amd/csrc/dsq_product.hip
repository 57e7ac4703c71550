// Products with a matrix that is held as messages (ds_product): y = x M^T, M's rows as 4-bit codes with a scale per block.
//
// Reading the message, 0.53 bytes a weight, is what cannot be done without, and leaves time for some four vector instructions a weight's
// share of a lane.  Codes are bytes after half an instruction each, so x is made of bytes, too, and the products are integers: per token
// and 128 columns ("chunk"; 64 where a block is 64), x = 2^e v with integers v of 16 bits (24 for fp32), written as two (three) signed bytes, which an
// i8 matrix instruction takes as rows of their own.  All sums inside a chunk are exact; 15 sum v, which takes codes 0 .. 15 to 2 code - 15, is where they start.  What is rounded is v:
// 2^-15 (2^-23) of the largest |x| next to it at most, which the same block's scale multiplies and no code drops, against the 2^-8 or 2^-11 of
// y's own rounding for 16-bit types (2^-24 for fp32).
//   A wave takes 16 (or 32) rows and a chunk at a time: lane (n, j) = (l % 16, l / 16) holds 32 codes of row n and the scale of its block, which is
// one factor for all of the lane's results.  x's bytes lie in LDS in the order in which codes come out of a word.
//   Three kernels.  One token: product_one_kernel.  Up to two matrix instructions of tokens (16; 8 for fp32), where reading codes is most of the work:
// product_tiles_kernel, whose workgroups make x's bytes themselves.  More tokens: product_kernel; a launch before makes x's bytes once, in work_dev,
// and codes go straight into registers, which leaves LDS to x.  Measured, us, product_tiles_kernel : product_kernel: 2 x 65536 x 4096, bf16,
// 34.0 : 62.0; 16 x 4096 x 16384, fp16, 19.4 : 26.7; 8 x 2048 x 2048 7.1 : 11.7; 4 x 16384 x 4096, fp32, 16.9 : 18.5; from there on 61 x 16001 x 4099,
// bf16, 55.7 : 38.6; 64 x 65536 x 1024 31.7 : 24.9, and in blocks of 64 51.4 : 31.6; 32 x 16384 x 4096, fp32, 30.3 : 26.9.
//   Where there are too few rows for the GPU, workgroups split the columns, too, and one more launch adds their sums.
#include "dsq_answers.h"
#include "dsq_codes.h"
#include "dsq_message_reads.h"

namespace dsq {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64, kChunk = 128;   // of a workgroup; columns a wave takes at a time
constexpr uint64_t kGroupsOfLaunch = 1u << 22;                    // a launch dimension holds fewer than 2^32 work-items

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// How x is written as bytes: `digits` rows of a matrix instruction per token, of which `stride` are set aside.
template <typename T>
struct Digits {
    static constexpr int digits = 2, stride = 2, exponent = 14;   // |v| <= 127 * 256 + 127, below 2^15
    static constexpr float most = 32639.f;
};
template <>
struct Digits<float> {
    static constexpr int digits = 3, stride = 4, exponent = 22;   // |v| <= 127 (2^16 + 2^8 + 1), below 2^23
    static constexpr float most = 8355711.f;
};
template <typename T>
constexpr int kTileTokens = 16 / Digits<T>::stride;               // tokens of a matrix instruction
template <typename T>
constexpr uint64_t kTokens = 8 * kTileTokens<T>;                  // of a launch
constexpr int kRowTiles = 2;                                      // of 16 rows, of a wave of product_kernel

struct ProductPlan {
    uint32_t parts, part_chunks;                                  // workgroups that split the columns, and the chunks (product_tiles_kernel: stages) of each
    uint32_t row_waves, wave_rows;                                // one token: waves side by side, the other kWaves / row_waves split the columns; rows of a wave
};

struct ProductShape : ProductArgs {
    ProductPlan plan;
    uint64_t row0;
    const uint8_t* panel;                                         // x as bytes, one record per chunk (see Record), or nullptr
    float* partial;                                               // parts x tokens x rows, or nullptr
};

// One chunk of x: the digits, [matrix instruction][j][row][16 columns]; the sums the products start from, -15 times the digits' sum, [block][row]
// (two blocks where a block is 64 columns); and per token what v counts, 2^e.  Rows: digit d of token t is row stride t + d; rows of no token hold anything.
template <typename T, int TT, bool NARROW>
struct Record {
    static constexpr uint32_t H = NARROW ? 2 : 1, rows = 16 * TT, sums = H * TT * 64, units = H * TT * 32, bytes = 128 * rows + sums + units;
    __device__ static i32x4* digits(uint8_t* r) { return reinterpret_cast<i32x4*>(r); }
    __device__ static int32_t* start(uint8_t* r) { return reinterpret_cast<int32_t*>(r + 128 * rows); }
    __device__ static float* unit(uint8_t* r) { return reinterpret_cast<float*>(r + 128 * rows + sums); }
};

// One weight after the other, as the formula has it: for a result that is not finite.
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
// The largest p for which 2^p x is below 2^(exponent + 1) and at most `limit`, of an |x| with these bits (not above 127: what is lost there is
// below 2^-127).
__device__ __forceinline__ int power_of(uint32_t bits, int exponent, float limit) {
    const int p = exponent + 127 - (int)(bits >> 23), q = p > 126 ? 126 : p;
    return __uint_as_float(bits) * power2_of(q) > limit ? q - 1 : q;
}

// op over 8 or 16 adjacent lanes, in all of them: each lane with its mirror image, then with the others of its four.
template <int CTRL>
__device__ __forceinline__ uint32_t other_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
template <int LANES, typename F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F op) {
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
// The bits of the largest of eight magnitudes, of the type's width; NaN is above all.  And the bits of the same number in fp32.
template <typename T>
__device__ __forceinline__ uint32_t largest_bits(typename EightOf<T>::Raw raw) {
    if constexpr (sizeof(T) == 2) {
        typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        const u16x8 bits = __builtin_bit_cast(u16x8, raw) & (uint16_t)0x7FFF;
        const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(bits.s01, bits.s23), __builtin_elementwise_max(bits.s45, bits.s67));
        return m.x > m.y ? m.x : m.y;
    } else {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = __float_as_uint((float)raw[e]) & 0x7FFFFFFFu;
            most = bits > most ? bits : most;
        }
        return most;
    }
}
template <typename T>
__device__ __forceinline__ uint32_t float_bits(uint32_t bits) {
    if constexpr (sizeof(T) == 2) return __float_as_uint((float)__builtin_bit_cast(T, (uint16_t)bits));
    else return bits;
}

// Sixteen adjacent lanes, lane u with columns 8 u .. 8 u + 7 of a chunk (raw), write a token's part of the chunk's record.
template <typename T, int TT, bool NARROW>
__device__ void make_digits(uint32_t tok, uint32_t u, typename EightOf<T>::Raw raw, uint8_t* record) {
    using D = Digits<T>;
    using R = Record<T, TT, NARROW>;
    constexpr int LANES = NARROW ? 8 : 16;                        // of a block
    // 2^power x, rounded, plus 128 in all digits but the highest: its bytes are the digits, their sign bits turned over where 128 was added
    uint32_t most = over_lanes<LANES>(largest_bits<T>(raw), [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    most = float_bits<T>(most);
    const int power = power_of(most, D::exponent, D::most);
    const bool finite = most < 0x7F800000u;                       // (if not, the block counts as NaN, whatever its digits are)
    const float to = power2_of(power);
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (D::digits == 2) v[e] = __float_as_uint(fmaf((float)raw[e], to, 12582912.f + 128.f));   // 1.5 2^23: an ulp is 1
        else v[e] = (uint32_t)(finite ? (int32_t)rintf((float)raw[e] * to) : 0) + 0x8080u;
    }
    uint32_t bytes[D::digits][2];                                 // the odd columns apart from the even ones
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        const uint32_t a = __builtin_amdgcn_perm(v[2 + o], v[o], 0x05010400u), b = __builtin_amdgcn_perm(v[6 + o], v[4 + o], 0x05010400u);
        bytes[D::digits - 1][o] = __builtin_amdgcn_perm(b, a, 0x05040100u) ^ 0x80808080u;
        bytes[D::digits - 2][o] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        if constexpr (D::digits == 3) {
            bytes[1][o] ^= 0x80808080u;
            const uint32_t c = __builtin_amdgcn_perm(v[2 + o], v[o], 0x0C0C0602u), d = __builtin_amdgcn_perm(v[6 + o], v[4 + o], 0x0C0C0602u);
            bytes[0][o] = __builtin_amdgcn_perm(d, c, 0x05040100u);
        }
    }
    const uint32_t t = NARROW ? u / 8 * 2 + u % 2 : u % 4, j = NARROW ? u % 8 / 2 : u / 4, rows = R::rows;
#pragma unroll
    for (int d = 0; d < D::digits; ++d) {
        const uint32_t at = (((t / 2) * 4 + j) * rows + tok * D::stride + d) * 16 + 8 * (t % 2);
        *reinterpret_cast<u32x2*>(record + at) = u32x2{bytes[d][0], bytes[d][1]};
        constexpr int kOff = (int)0xF1F1F1F1;                     // -15 each
        const int32_t sum = __builtin_amdgcn_sdot4((int)bytes[d][0], kOff, __builtin_amdgcn_sdot4((int)bytes[d][1], kOff, 0, false), false);
        const uint32_t total = over_lanes<LANES>((uint32_t)sum, [](uint32_t x, uint32_t y) { return x + y; });
        if (u % LANES == 0) R::start(record)[u / LANES * (TT * 16) + tok * D::stride + d] = (int32_t)total;
    }
    if (u % LANES == 0) R::unit(record)[u / LANES * (TT * 8) + tok] = finite ? power2_of(-power) : __builtin_nanf("");
}

// x as bytes, for all workgroups: 16 threads per chunk and token.
template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(256) product_digits_kernel(ProductShape a, uint8_t* panel) {
    const uint64_t chunk = blockIdx.x;
    const uint32_t tok = threadIdx.x / 16 + 16 * blockIdx.y, u = threadIdx.x % 16;
    if (tok >= a.tokens) return;
    const T* x = static_cast<const T*>(a.in) + tok * a.in_ld;
    make_digits<T, TT, NARROW>(tok, u, load_eight(x, (uint32_t)chunk * kChunk + 8 * u, (uint32_t)a.cols), panel + chunk * Record<T, TT, NARROW>::bytes);
}

// The products of a chunk of codes, 16 RT rows, with the chunk's record of x.
template <typename T, int TT, int RT, bool NARROW>
__device__ __forceinline__ void multiply(const Codes<NARROW> (&c)[RT], uint8_t* rec, uint32_t n, uint32_t j,
                                         float (&sum)[RT][TT][4 / Digits<T>::stride]) {
    using D = Digits<T>;
    using R = Record<T, TT, NARROW>;
    constexpr int H = NARROW ? 2 : 1, PER = 4 / D::stride;        // blocks of a chunk; tokens of a lane and matrix instruction
    const i32x4* digits = R::digits(rec);
    i32x4 codes[RT][2];
    float unit[RT][H];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            codes[r][h] = i32x4{(int)(c[r].w[2 * h] << 1 & 0x1E1E1E1Eu), (int)(c[r].w[2 * h] >> 3 & 0x1E1E1E1Eu),
                                (int)(c[r].w[2 * h + 1] << 1 & 0x1E1E1E1Eu), (int)(c[r].w[2 * h + 1] >> 3 & 0x1E1E1E1Eu)};
#pragma unroll
        for (int b = 0; b < H; ++b) unit[r][b] = c[r].scale[b] * (1.f / 15.f);
    }
    struct Left {
        i32x4 x[2], start[H];
        float count[H][PER];
    };
    auto load = [&](Left& v, int t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) v.x[h] = digits[(4 * h + j) * R::rows + 16 * t + n];
#pragma unroll
        for (int b = 0; b < H; ++b) {
#pragma unroll
            for (int i = 0; i < PER; ++i) v.count[b][i] = R::unit(rec)[b * (TT * 8) + (4 * t + j) * PER + i];
            v.start[b] = *reinterpret_cast<const i32x4*>(R::start(rec) + b * (TT * 16) + 16 * t + 4 * j);
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
                i32x4 p;
                if constexpr (NARROW) {
                    p = __builtin_amdgcn_mfma_i32_16x16x64_i8(v.x[b], codes[r][b], v.start[b], 0, 0, 0);
                } else {
                    p = __builtin_amdgcn_mfma_i32_16x16x64_i8(v.x[0], codes[r][0], v.start[0], 0, 0, 0);
                    p = __builtin_amdgcn_mfma_i32_16x16x64_i8(v.x[1], codes[r][1], p, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    float w;
                    if constexpr (D::digits == 2) w = (float)((p[2 * i] << 8) + p[2 * i + 1]);
                    else w = fmaf(fmaf((float)p[0], 256.f, (float)p[1]), 256.f, (float)p[2]);
                    sum[r][t][i] = fmaf(unit[r][b] * v.count[b][i], w, sum[r][t][i]);
                }
            }
        if constexpr (TT > 2) {                                   // what is asked for, and what is left to do, beyond the next tile takes registers
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < PER; ++i) asm volatile("" : "+v"(sum[r][t][i]));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// More tokens: a workgroup takes 256 rows, chunk after chunk, its waves 32 rows each against the same x in LDS.  61 x 16001 x 4099, bf16, in blocks of 64: 30 us;
// for every token, row and block four vector instructions, 45 % of the clocks, and the matrix instructions 15 %.
template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(kThreads) product_kernel(ProductShape a) {
    constexpr int RT = kRowTiles;
    using R = Record<T, TT, NARROW>;
    constexpr int PER = 4 / Digits<T>::stride;                    // tokens of a lane and matrix instruction
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
    auto use = [&](const Codes<NARROW> (&codes)[RT], uint32_t c) { multiply<T, TT, RT, NARROW>(codes, lds + (c & 1) * record, n, j, sum); };
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
// gathers scales alone costs the memory pipeline as much as one that brings 16 bytes a lane (2 x 65536 x 4096, blocks of 256, 34.0 us, 42.9 with scales read
// apart; 16 x 4096 x 16384, where the instructions count, 19.4 and 18.8).  Blocks of more than 256 columns are read in eight pieces, and their scales once a
// block (of 2048: 30.2 us).
//   2 tokens of 65536 x 4096 read 4.2 TB/s.  16 tokens cost some 340 instructions a stage, 5400 clocks for the two workgroups of a compute unit, in which it
// could read 44 KB and reads 32: x's digits are a third of them; 44.2 us, and 2.3 TB/s for 16 x 4096 x 16384, whose workgroups have four stages each.
// Slower: two stages ahead (registers; 16 x 4096 x 16384 22.8 us), workgroups of 256 rows (2 x 65536 x 4096 46.8 : 42.9).
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
    constexpr int PER = 4 / Digits<T>::stride;
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
        if (x_tok < tokens) make_digits<T, TT, NARROW>(x_tok, x_unit % 16, v.x, records + x_unit / 16 * record);
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
            multiply<T, TT, 1, NARROW>(codes, half_at + S::codes + S::scales + c * record, n, j, sum);
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
// registers.  A lane keeps 32 columns of x for all the rows of its wave, G lanes hold a row, and a load takes 64 / G rows of 32 G columns.  x is
// written in digits of four bits here, 16^d apart, 4 of them (6 for fp32), with an exponent per 32 columns: eight codes (less 8, so that they are
// signed) meet eight digits in one instruction, 0.6 instructions a weight.  The lanes of a row are joined by a tree of lane shifts.  65536 x 4096: 24.6 us,
// 5.8 TB/s, the vector units busy 67 % of the time.
constexpr uint32_t kLaneCols = 32;
template <typename T>
struct Nibbles {
    static constexpr int digits = 4, exponent = 14;
    static constexpr float most = 30583.f;                        // 7 (16^3 + 16^2 + 16 + 1)
};
template <>
struct Nibbles<float> {
    static constexpr int digits = 6, exponent = 22;
    static constexpr float most = 7829367.f;
};

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

template <typename T, int G>
__global__ void __launch_bounds__(kThreads) product_one_kernel(ProductShape a) {
    using D = Nibbles<T>;
    constexpr int AT_ONCE = 64 / G, AHEAD = 4;                    // rows of a load, loads under way
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), g = lane / G, l = lane % G;
    const uint32_t row_waves = a.plan.row_waves, col_waves = kWaves / row_waves, rw = wave % row_waves, cw = wave / row_waves;
    const uint32_t wave_rows = a.plan.wave_rows, rows_here = row_waves * wave_rows, loads = wave_rows / AT_ONCE;
    const uint64_t first = a.row0 + (uint64_t)blockIdx.x * rows_here;
    const uint32_t block_log2 = 31 - __builtin_clz(a.block);
    const uint32_t lanes = col_waves * G;                         // lanes that hold different columns ...
    i32x4* digits = reinterpret_cast<i32x4*>(lds);                // ... and their digits, [digit][lane]; then sum v and what v counts
    int32_t* sums = reinterpret_cast<int32_t*>(digits + D::digits * lanes);
    float* units = reinterpret_cast<float*>(sums + lanes);
    float* totals = units + lanes;                                // [column wave][row of the workgroup]
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

        // the workgroup writes this stretch of x in digits: a thread takes eight columns, four threads a lane's 32
        if (slice) __syncthreads();
        for (uint32_t w = threadIdx.x; w < lanes * 4; w += kThreads) {
            const uint64_t at = slice + 8 * w;
            float v[8];
            if (at + 8 <= a.cols) {
                typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
                const Raw raw = *reinterpret_cast<const Raw*>(x + at);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (float)raw[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = at + e < a.cols ? (float)x[at + e] : 0.f;
            }
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t bits = __float_as_uint(v[e]) & 0x7FFFFFFFu;
                most = bits > most ? bits : most;
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                const uint32_t other = (uint32_t)__shfl_xor((int)most, o);
                most = other > most ? other : most;
            }
            const int power = power_of(most, D::exponent, D::most);
            const bool finite = most < 0x7F800000u;
            const float to = power2_of(power);
            uint32_t out[D::digits];
            int32_t sum = 0;
#pragma unroll
            for (int d = 0; d < D::digits; ++d) out[d] = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                int32_t rest = finite ? (int32_t)rintf(v[e] * to) : 0;
                sum += rest;
#pragma unroll
                for (int d = 0; d < D::digits; ++d) {             // the first digit is the lowest; signed, [-8, 7]
                    const int32_t digit = rest << 28 >> 28;
                    rest = (rest - digit) >> 4;
                    out[d] |= ((uint32_t)digit & 15u) << (4 * e);
                }
            }
            const uint32_t place = (w % 4 + missing_words(slice + w / 4 * kLaneCols, a.cols)) % 4;
#pragma unroll
            for (int d = 0; d < D::digits; ++d) reinterpret_cast<uint32_t*>(digits + d * lanes + w / 4)[place] = out[d];
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) sum += __shfl_xor(sum, o);
            if (w % 4 == 0) {
                sums[w / 4] = sum;
                units[w / 4] = finite ? power2_of(-power) * (1.f / 15.f) : __builtin_nanf("");
            }
        }
        __syncthreads();
        i32x4 own[D::digits];
#pragma unroll
        for (int d = 0; d < D::digits; ++d) own[d] = digits[d * lanes + cw * G + l];
        const int32_t start = sums[cw * G + l];
        const float unit = units[cw * G + l];

        auto use = [&](const Load& v, uint32_t q) {
            int32_t codes[4], dot[D::digits];
#pragma unroll
            for (int w = 0; w < 4; ++w) codes[w] = (int32_t)(v.w[w] ^ 0x88888888u);         // code - 8
#pragma unroll
            for (int d = 0; d < D::digits; ++d) {
                dot[d] = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) dot[d] = __builtin_amdgcn_sdot8(codes[w], own[d][w], dot[d], false);
            }
            float sum;                                            // sum (2 code - 15) v = 2 sum (code - 8) v + sum v
            if constexpr (D::digits == 4) {
                sum = (float)(2 * ((((dot[3] * 16 + dot[2]) * 16 + dot[1]) * 16) + dot[0]) + start);
            } else {
                const int32_t high = (dot[5] * 16 + dot[4]) * 16 + dot[3], low = (dot[2] * 16 + dot[1]) * 16 + dot[0];
                sum = fmaf((float)high, 8192.f, (float)(2 * low + start));
            }
            sum = lanes_total<G>((some ? v.scale : 0.f) * unit * sum);
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
    if (tiles <= 2) {
        // Two workgroups for every compute unit where each has four stages, otherwise one where it has any: 4 x 16384 x 4096, fp32, 2 parts (256 workgroups)
        // 17.6 us, 4: 16.2, 6: 16.8; 16 x 20000 x 4096, bf16, blocks of 64, 1 part (157) 26.0, 3: 24.0; 16 x 4096 x 4096 4 parts (128) 14.1, 8 (of two stages)
        // 10.6, 16: 12.6; 16 x 5000 x 4096 6 parts (240) 13.2, 12: 14.5; 8 x 2048 x 2048 1 part 9.6, 8 (128 workgroups, a stage each): 7.1.
        const uint64_t stages = (chunks + kStageChunks - 1) / kStageChunks, groups = (rows + 16 * kWaves - 1) / (16 * kWaves);
        p.parts = split(512, groups, stages);
        if (stages < 4 * p.parts) p.parts = split(256, groups, stages);
        if (stages < 6) p.parts = 1;                              // (a stage takes 0.76 us where there are few workgroups, the launch that joins 2.6)
        p.part_chunks = (uint32_t)((stages + p.parts - 1) / p.parts);
        p.parts = (uint32_t)((stages + p.part_chunks - 1) / p.part_chunks);
        return p;
    }
    const uint64_t height = 16 * kRowTiles * kWaves, groups = (rows + height - 1) / height;
    // Workgroups split the columns until all compute units have one, and not one more, which would take as long again or add to what is joined: 61 x 16001 x
    // 4099, bf16, 4 parts (252 workgroups) 39.1 us, 8: 48.3; 64 x 65536 x 1024 1 part (256) 25.7, 2: 41.5; 64 x 2048 x 2048, fp32, 4 parts (of four chunks) 14.5,
    // 16 (128 workgroups, a chunk each) 11.8; 30 x 300 x 1000, bf16, 2 parts 12.7, 8: 10.8.
    p.parts = chunks < 4 ? 1 : split(256, groups, chunks);        // (a chunk takes a microsecond where there are few workgroups, the launch that joins 2.6)
    p.part_chunks = (uint32_t)((chunks + p.parts - 1) / p.parts);
    p.parts = (uint32_t)((chunks + p.part_chunks - 1) / p.part_chunks);
    return p;
}

// product_one_kernel's calls: a row has four words.
bool by_rows(uint64_t tokens, uint64_t cols) { return tokens == 1 && cols > 24; }

// Scratch: the panel (of product_kernel), then the partial sums.
template <typename T>
uint64_t panel_bytes(uint64_t cols, uint64_t tokens, bool narrow) {
    return product_tiles<T>(tokens) > 2 ? (cols + kChunk - 1) / kChunk * record_bytes<T>(tokens, narrow) : 0;
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
    if constexpr (TT <= 2) {
        launch_product_tiles<T, TT, NARROW>(a, stream);
    } else {
        constexpr uint32_t lds = 2 * Record<T, TT, NARROW>::bytes;
        static_assert(lds <= 64 * 1024, "what a launch may ask for");
        hipLaunchKernelGGL((product_digits_kernel<T, TT, NARROW>), dim3((unsigned)((a.cols + kChunk - 1) / kChunk), (unsigned)(a.tokens + 15) / 16), dim3(256), 0, stream, a,
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
    // Rows enough to be worth writing x in digits for, as long as there is a workgroup for every compute unit: 65536 x 4096, bf16, 8 rows a wave 32.6 us,
    // 16: 27.9, 32: 28.2, 64: 28.6; 4096 x 16384 8: 15.4 (512 workgroups), 16: 13.2, 32: 16.8 (128); 2048 x 2048 1: 4.1, 4: 4.7, 16: 7.6.
    const uint64_t each = a.rows / (256ull * a.plan.row_waves) / AT_ONCE * AT_ONCE;
    a.plan.wave_rows = (uint32_t)(each < AT_ONCE ? AT_ONCE : each > 32 ? 32 : each);
    const uint64_t rows_here = (uint64_t)a.plan.row_waves * a.plan.wave_rows;
    const uint32_t bytes = col_waves * G * (Nibbles<T>::digits * 16 + 8) + kWaves * a.plan.wave_rows * 4;
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
