// Products with a matrix that is held as messages (ds_product): y = x M^T, M's rows as 4-bit codes with a scale per block.
//
// What bounds it is reading the message, 0.53 bytes a weight, as long as 64 tokens or fewer share it.  So the codes go
// straight from memory into matrix instructions: a wave takes 16 (or 32) rows and 128 columns at a time, lane l holds 32 codes of row
// l % 16 (one 16-byte load) and its block's scale, and each word of eight codes becomes an operand with eight instructions (dsq_codes.h).  With the tokens as
// the other operand a lane's results all belong to its own row, so the block's scale is one factor per lane.
//   x is laid out once per workgroup, in LDS, as the operands need it: units of eight columns in the order in which a word's codes come
// out, zero behind the last column.  The waves of a workgroup share it; they split its rows, and, where there are few rows, its columns,
// too (joined in LDS).  Columns are also split over workgroups where x does not fit into LDS; then fp32 partial sums go through work_dev and a
// second launch adds them, in the order of the columns.
#include "dsq_answers.h"
#include "dsq_codes.h"

namespace dsq {
namespace {

constexpr int kWaves = 8, kChunk = 128;                           // waves of a workgroup; columns a wave takes at a time
constexpr uint32_t kPanel = 64 * 1024;                            // bytes of LDS for x: two workgroups fit on a compute unit
constexpr uint64_t kTokens = 64;                                  // of a launch
constexpr uint64_t kGroupsOfLaunch = 1u << 22;                    // a launch dimension holds fewer than 2^32 work-items

struct ProductPlan {
    uint32_t row_waves;                                           // waves side by side; the other kWaves / row_waves split the columns
    uint32_t parts, part_chunks;                                  // workgroups that split the columns, and the chunks of each
    uint32_t panel_chunks;                                        // chunks of x that are in LDS at a time
};

struct ProductShape : ProductArgs {
    ProductPlan plan;
    uint64_t row0;
    float* partial;                                               // parts x tokens x rows, or nullptr
};

// One weight after the other, as the formula has it: for a result that is not finite.
template <typename T>
__device__ __noinline__ float product_in_order(const ProductArgs& a, uint64_t r, uint64_t t) {
    const uint8_t* row = a.msg + r * a.row_bytes;
    const T* x = static_cast<const T*>(a.in) + t * a.in_ld;
    const uint32_t per = a.block / 8;
    float sum = 0.f;
    for (uint64_t w = 0; 8 * w < a.cols; ++w) {
        const uint8_t* block = row + w / per * (4 + a.block / 2);
        const float unit = *reinterpret_cast<const float*>(block) * (16.f / 15.f);
        const uint32_t word = *reinterpret_cast<const uint32_t*>(block + 4 + 4 * (w % per));
        float part = 0.f;                                         // a code counts as (2 code - 15) / 16: no sum is infinite before y is
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
// Word t goes with words t of the other lanes of the row, lanes j = 0 .. 3, into one matrix instruction, and instructions must not mix blocks:
// word t of lane j starts at column 32 j + 8 t, or at 64 floor(t / 2) + 16 j + 8 (t % 2) where a block is 64 columns.
template <bool NARROW>
struct Codes {
    uint32_t w[4];
    float scale[NARROW ? 2 : 1];
};
template <bool NARROW>
__device__ __forceinline__ uint32_t word_column(uint32_t t, uint32_t j) { return NARROW ? 64 * (t / 2) + 16 * j + 8 * (t % 2) : 32 * j + 8 * t; }
// ... and the other way: (t, j) of the eight columns that start at 8 u.
template <bool NARROW>
__device__ __forceinline__ uint32_t column_place(uint32_t u) { return NARROW ? (u / 8 * 2 + u % 2) * 4 + u % 8 / 2 : u % 4 * 4 + u / 4; }

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

template <typename T, int TT, int RT, bool NARROW>
__global__ void __launch_bounds__(kWaves * 64, 2) product_kernel(ProductShape a) {
    using O = typename Operand<T>::type;
    constexpr int P = Operand<T>::pieces;
    extern __shared__ __align__(16) uint8_t lds[];
    Eight<O>* panel = reinterpret_cast<Eight<O>*>(lds);           // [chunk][t][piece][j][token]
    const uint32_t tokens = (uint32_t)a.tokens;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, n = lane & 15, j = lane >> 4;
    const uint32_t row_waves = a.plan.row_waves, col_waves = kWaves / row_waves;
    const uint32_t rw = wave % row_waves, cw = wave / row_waves;
    const uint64_t c0 = (uint64_t)blockIdx.y * a.plan.part_chunks, all_chunks = (a.cols + kChunk - 1) / kChunk;
    const uint32_t chunks = (uint32_t)(all_chunks - c0 < a.plan.part_chunks ? all_chunks - c0 : a.plan.part_chunks);
    const uint32_t block_log2 = 31 - __builtin_clz(a.block);

    const uint64_t first = a.row0 + ((uint64_t)blockIdx.x * row_waves + rw) * (16 * RT);
    const uint8_t* row[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {                                // rows behind the last read the last one, and are not stored
        const uint64_t at = first + 16 * r + n;
        row[r] = a.msg + (at < a.rows ? at : a.rows - 1) * a.row_bytes;
    }
    uint32_t tok_at[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) tok_at[t] = 16 * t + n < tokens ? 16 * t + n : tokens - 1;
    f32x4 sum[RT][TT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) sum[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto use = [&](const Codes<NARROW> (&c)[RT], uint32_t chunk) {
#pragma unroll
        for (int h = 0; h < (NARROW ? 2 : 1); ++h) {
            f32x4 part[RT][TT];
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                f32x4 off = {0.f, 0.f, 0.f, 0.f};
                constexpr int words = NARROW ? 2 : 4;
#pragma unroll
                for (int w = 0; w < words; ++w)
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        off = matrix_fma(panel[(((chunk * 4 + h * words + w) * P + p) * 4 + j) * tokens + tok_at[t]], centre_operand<O>(), off);
                off = -off;
#pragma unroll
                for (int r = 0; r < RT; ++r) part[r][t] = off;
            }
#pragma unroll
            for (int w = 0; w < (NARROW ? 2 : 4); ++w) {
                Eight<O> codes[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) codes[r] = code_operand<O>(c[r].w[(NARROW ? 2 * h : 0) + w]);
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int t = 0; t < TT; ++t) {
                        const Eight<O> x = panel[(((chunk * 4 + (NARROW ? 2 * h : 0) + w) * P + p) * 4 + j) * tokens + tok_at[t]];
#pragma unroll
                        for (int r = 0; r < RT; ++r) part[r][t] = matrix_fma(x, codes[r], part[r][t]);
                    }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float unit = c[r].scale[h] * kPerCode;
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[r][t][i] = fmaf(unit, part[r][t][i], sum[r][t][i]);
            }
        }
    };
    // x goes through LDS in stages of panel_chunks; codes of the next chunks are under way while these are multiplied
    constexpr int AHEAD = 2;
    Codes<NARROW> ring[AHEAD][RT];
    for (uint32_t from = 0; from < chunks; from += a.plan.panel_chunks) {
        const uint32_t count = chunks - from < a.plan.panel_chunks ? chunks - from : a.plan.panel_chunks;
        const uint64_t col0 = (c0 + from) * kChunk;
        const uint32_t whole = (uint32_t)(a.cols / kChunk - (c0 + from) < count ? a.cols / kChunk - (c0 + from) : count);   // chunks without a ragged end
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
            if (cw + s * col_waves < whole)
#pragma unroll
                for (int r = 0; r < RT; ++r) load_codes<NARROW>(ring[s][r], row[r], block_log2, col0 + (uint64_t)(cw + s * col_waves) * kChunk, j);
        if (from) __syncthreads();
        // x as operands: a thread takes eight columns of a token at a time
        for (uint32_t q = threadIdx.x; q < count * 16 * tokens; q += kWaves * 64) {
            const uint32_t tok = q / (count * 16), u = q % (count * 16);
            const uint64_t col = (c0 + from) * kChunk + 8 * u;
            const T* x = static_cast<const T*>(a.in) + tok * a.in_ld + col;
            float v[8];
            if (col + 8 <= a.cols) {
                typedef T Raw __attribute__((ext_vector_type(8), aligned(sizeof(T))));
                const Raw raw = *reinterpret_cast<const Raw*>(x);
    #pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (float)raw[e / 2 + 4 * (e % 2)];
            } else {
    #pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = col + e / 2 + 4 * (e % 2) < a.cols ? (float)x[e / 2 + 4 * (e % 2)] : 0.f;
            }
            Eight<O> out[P];
            split_operand<O, P>(v, out);
            const uint32_t place = column_place<NARROW>(u % 16), base = (u / 16 * 4 + place / 4) * P;
    #pragma unroll
            for (int p = 0; p < P; ++p) panel[((base + p) * 4 + place % 4) * tokens + tok] = out[p];
        }
        __syncthreads();
        for (uint32_t c = cw; c < whole; c += AHEAD * col_waves) {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const uint32_t here = c + s * col_waves;
                if (here >= whole) break;
                Codes<NARROW> now[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) now[r] = ring[s][r];
                if (here + AHEAD * col_waves < whole)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        load_codes<NARROW>(ring[s][r], row[r], block_log2, col0 + (uint64_t)(here + AHEAD * col_waves) * kChunk, j);
                use(now, here);
            }
        }
        if (whole < count && whole % col_waves == cw) {
            Codes<NARROW> now[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) load_codes_tail<NARROW>(now[r], row[r], block_log2, col0 + (uint64_t)whole * kChunk, a.cols, j);
            use(now, whole);
        }
    }

    // the waves that split the columns: join in LDS
    if (col_waves > 1) {
        __syncthreads();
        f32x4* joined = reinterpret_cast<f32x4*>(lds);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t) joined[((wave * RT + r) * TT + t) * 64 + lane] = sum[r][t];
        __syncthreads();
        if (cw != 0) return;
        for (uint32_t c = 1; c < col_waves; ++c)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int t = 0; t < TT; ++t) sum[r][t] += joined[(((c * row_waves + rw) * RT + r) * TT + t) * 64 + lane];
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t at = first + 16 * r + n;
                const uint32_t tok = 16 * t + 4 * j + i;
                if (at >= a.rows || tok >= tokens) continue;
                if (a.partial) a.partial[((uint64_t)blockIdx.y * tokens + tok) * a.rows + at] = sum[r][t][i];
                else product_store<T>(a, at, tok, sum[r][t][i]);
            }
}

// Adds the parts.  A thread per row and token.
template <typename T>
__global__ void __launch_bounds__(256) product_join_kernel(ProductShape a) {
    const uint64_t r = a.row0 + (uint64_t)blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
    if (r >= a.rows) return;
    float v = 0.f;
    for (uint32_t p = 0; p < a.plan.parts; ++p) v += a.partial[(p * a.tokens + t) * a.rows + r];
    product_store<T>(a, r, t, v);
}

template <typename T>
uint32_t panel_bytes_of_chunk(uint64_t tokens) { return (uint32_t)(tokens * kChunk * 2 * Operand<T>::pieces); }

uint32_t rows_of_wave(uint64_t tokens) { return tokens > 16 ? 32 : 16; }

template <typename T>
ProductPlan product_plan(uint64_t rows, uint64_t cols, uint64_t tokens) {
    ProductPlan p{};
    const uint64_t chunks = (cols + kChunk - 1) / kChunk, tiles = (rows + rows_of_wave(tokens) - 1) / rows_of_wave(tokens);
    // A workgroup reads all of x for the rows it has: not more bytes of it than of codes, as far as eight waves of rows go.
    p.row_waves = 1;
    while (p.row_waves < kWaves && (tokens * 4 * Operand<T>::pieces > rows_of_wave(tokens) * p.row_waves || tiles / (2 * p.row_waves) >= 512)) p.row_waves *= 2;
    const uint64_t groups = (tiles + p.row_waves - 1) / p.row_waves, col_waves = kWaves / p.row_waves;
    p.parts = 1;
    while (groups * p.parts < 256 && chunks >= 8 * p.parts * col_waves && p.parts < 32) p.parts *= 2;
    p.part_chunks = (uint32_t)((chunks + p.parts - 1) / p.parts);
    p.parts = (uint32_t)((chunks + p.part_chunks - 1) / p.part_chunks);
    const uint32_t fit = kPanel / panel_bytes_of_chunk<T>(tokens);
    p.panel_chunks = p.part_chunks < fit ? p.part_chunks : fit;
    return p;
}

template <typename T, int TT, int RT, bool NARROW>
void launch_product_kernel(const ProductShape& a, hipStream_t stream) {
    const uint32_t join = a.plan.row_waves == kWaves ? 0 : kWaves * RT * TT * 64 * 16;
    const uint32_t panel = a.plan.panel_chunks * panel_bytes_of_chunk<T>(a.tokens), bytes = panel > join ? panel : join;
    const uint64_t groups = (a.rows + 16 * RT * a.plan.row_waves - 1) / (16 * RT * a.plan.row_waves);
    ProductShape b = a;
    for (uint64_t g = 0; g < groups; g += kGroupsOfLaunch) {
        b.row0 = g * 16 * RT * a.plan.row_waves;
        const uint64_t here = groups - g < kGroupsOfLaunch ? groups - g : kGroupsOfLaunch;
        hipLaunchKernelGGL((product_kernel<T, TT, RT, NARROW>), dim3((unsigned)here, a.plan.parts), dim3(kWaves * 64), bytes, stream, b);
    }
}

template <typename T>
void launch_product_of(const ProductArgs& args, hipStream_t stream) {
    for (uint64_t t0 = 0; t0 < args.tokens; t0 += kTokens) {
        ProductShape a{};
        static_cast<ProductArgs&>(a) = args;
        a.tokens = args.tokens - t0 < kTokens ? args.tokens - t0 : kTokens;
        a.in = static_cast<const T*>(args.in) + t0 * args.in_ld;
        a.out = static_cast<T*>(args.out) + t0 * args.out_ld;
        a.plan = product_plan<T>(a.rows, a.cols, a.tokens);
        a.partial = a.plan.parts > 1 ? static_cast<float*>(a.work) : nullptr;
        const bool narrow = a.block == 64;
        if (a.tokens <= 16) narrow ? launch_product_kernel<T, 1, 1, true>(a, stream) : launch_product_kernel<T, 1, 1, false>(a, stream);
        else if (a.tokens <= 32) narrow ? launch_product_kernel<T, 2, 2, true>(a, stream) : launch_product_kernel<T, 2, 2, false>(a, stream);
        else narrow ? launch_product_kernel<T, 4, 2, true>(a, stream) : launch_product_kernel<T, 4, 2, false>(a, stream);
        if (!a.partial) continue;
        const uint64_t groups = (a.rows + 255) / 256;
        for (uint64_t g = 0; g < groups; g += kGroupsOfLaunch) {
            a.row0 = g * 256;
            const uint64_t here = groups - g < kGroupsOfLaunch ? groups - g : kGroupsOfLaunch;
            hipLaunchKernelGGL(product_join_kernel<T>, dim3((unsigned)here, (unsigned)a.tokens), dim3(256), 0, stream, a);
        }
    }
}

}  // namespace

uint64_t product_work_bytes(const ds_matrix& m) {
    const uint64_t tokens = m.tokens < kTokens ? m.tokens : kTokens;
    uint64_t parts = 1;
    uint64_t bytes = 0;
    auto most = [&](uint64_t of) {                                // of the launches: whole ones and the last
        by_dtype(m.dtype, [&](auto kind) { parts = product_plan<decltype(kind)>(m.rows, m.cols, of).parts; });
        const uint64_t here = parts > 1 ? parts * of * m.rows * sizeof(float) : 0;
        if (here > bytes) bytes = here;
    };
    most(tokens);
    if (m.tokens % kTokens) most(m.tokens % kTokens);
    return bytes;
}

hipError_t launch_product(const ProductArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_product_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
