// The gradient of ds_product with respect to its vectors (ds_product_gradient): dx = dy M, M's rows as 4-bit codes with a scale per block.
//
// The sum runs over the matrix's rows, so the scales belong to what is summed: dy * scale is the other operand, made anew for every block
// of columns and rounded to bf16 pieces (two for 16-bit dtypes, 2^-17 relative, three for fp32: 24 bits; the smallest bf16 is 2^-133).  A wave takes 128 columns and 32
// rows at a time: lane (n, j) loads word n (eight columns) of rows 8 j .. 8 j + 7, and column c of all words, c = 0 .. 7, is one matrix
// instruction: codes of two rows sit in the halves of a register after one byte permutation, two more instructions make operands of two (dsq_codes.h).
// The waves of a workgroup and the workgroups of a column take different rows; the waves join in LDS, the workgroups through fp32 partial sums in
// work_dev and a second launch.
//   64 tokens of 32768 x 4096, bf16: 46.2 us, 1.5 TB/s of codes, where reading them takes 13.  Of a compute unit's 5200 clocks for 256 rows the matrix units
// work 2300 and the vector units 2700, more than half of it on dy * scale, of which every 128 columns need their own: two waves fit on a SIMD and hide a part
// of one behind the other.  Loads of a step that were all asked for at its start held up the eight waves for some 2000 clocks; next to the products they do not.
#include "dsq_answers.h"
#include "dsq_codes.h"

namespace dsq {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64, kChunk = 128, kStep = 32;   // of a workgroup; columns and rows a wave takes at a time
constexpr uint32_t kBlockRows = kWaves * kStep;                   // rows the workgroup takes at a time
// Tokens of a launch: what a wave has registers for.
template <typename T>
constexpr uint64_t kTokens(bool narrow) { return sizeof(T) == 4 || narrow ? 32 : 64; }
constexpr uint64_t kGroupsOfLaunch = 1u << 22;                    // a launch dimension holds fewer than 2^32 work-items

struct GradientShape : ProductArgs {
    uint32_t parts;                                               // workgroups that split the rows
    uint64_t part_rows;                                           // a multiple of kBlockRows
    uint64_t chunks, chunk0;
    float* partial;                                               // parts x tokens x cols, or nullptr
};

// One weight after the other, as the formula has it: for a result that is not finite.  A thread goes through the column by itself, up to the first NaN:
// 32768 x 4096, bf16, an infinity in a token's last place, 11 ms, for one token as for 64.
template <typename T>
__device__ __forceinline__ float gradient_in_order(const ProductArgs& a, uint64_t c, uint64_t t) {
    const uint8_t* block = a.msg + c / a.block * (4 + a.block / 2);
    const uint32_t at = c % a.block / 8, by = c % 8 * 4;
    const T* dy = static_cast<const T*>(a.in) + t * a.in_ld;
    float sum = 0.f;
#pragma unroll 1
    for (uint64_t r = 0; r < a.rows; ++r, block += a.row_bytes) {
        const float d = (float)dy[r] * (*reinterpret_cast<const float*>(block) / 15.f);
        const uint32_t word = *reinterpret_cast<const uint32_t*>(block + 4 + 4 * at);
        sum = fmaf((float)(2 * (int)(word >> by & 15u) - 15), d, sum);
        if (sum != sum) break;                                    // and NaN stays
    }
    return sum;
}

template <typename T>
__device__ __forceinline__ void gradient_store(const ProductArgs& a, uint64_t c, uint64_t t, float v) {
    if (!(fabsf(v) < __builtin_huge_valf())) v = gradient_in_order<T>(a, c, t);
    static_cast<T*>(a.out)[t * a.out_ld + c] = (T)v;
}

// What a wave needs of the matrix in 32 rows.  A matrix instruction's columns must share a block: with blocks of 64 a lane takes four columns of either
// block, half of word n / 2, and its column c is 64 floor(c / 4) + 4 n + c % 4 instead of 8 n + c.
template <bool NARROW>
struct Rows {
    static constexpr int H = NARROW ? 2 : 1;
    uint32_t w[H][8];
    float scale[H][8];
};

template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(kThreads, 2) product_gradient_kernel(GradientShape a) {
    constexpr int P = sizeof(T) == 4 ? 3 : 2, H = NARROW ? 2 : 1;
    // What codes are too large by is taken off at the end, or, for fp32, every 32 rows, before sums grow: they are five times what the difference is, and so were
    // their roundings (8192 x 5000, 16 tokens: 1.7e-6 of the result, now 8.5e-7, as sums in fp32 have).
    constexpr bool kCentred = sizeof(T) == 4;
    constexpr uint32_t E = 16 / sizeof(T), PER = kBlockRows / E, PIECES = TT * 16 * PER / kThreads;   // 16-byte pieces of dy: elements, of a token, of a thread
    constexpr uint32_t kPitch = kBlockRows + E;                   // of a token's dy in LDS, elements
    using R = Rows<NARROW>;
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    typedef T Eights __attribute__((ext_vector_type(8), aligned(16)));
    extern __shared__ __align__(16) uint8_t lds[];
    T* staged = reinterpret_cast<T*>(lds);                        // [buffer][token][row]
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = lane & 15, j = lane >> 4;
    const uint32_t tokens = (uint32_t)a.tokens;
    // Workgroups go round the eight XCDs: those of the same rows, which share cache lines, onto one of them.
    const uint64_t id = (uint64_t)blockIdx.y * gridDim.x + blockIdx.x, all = (uint64_t)gridDim.x * gridDim.y;
    const uint64_t xcd = id % 8, mine = xcd * (all / 8) + (xcd < all % 8 ? xcd : all % 8) + id / 8;
    const uint64_t chunk = mine % gridDim.x, part = mine / gridDim.x;
    const uint64_t col0 = (a.chunk0 + chunk) * kChunk;
    const uint64_t r_begin = part * a.part_rows, r_end = r_begin + a.part_rows < a.rows ? r_begin + a.part_rows : a.rows;
    const uint32_t blocks = (uint32_t)((r_end - r_begin + kBlockRows - 1) / kBlockRows);

    const uint32_t pitch = 4 + a.block / 2;
    const uint8_t* block[H];                                      // in row 0: the blocks, and the lane's word in them
    uint32_t at[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const uint64_t col = col0 + 64 * h, mine = NARROW ? col + n / 2 * 8 : col + 8 * n;
        block[h] = a.msg + (col < a.cols ? col : 0) / a.block * pitch;
        at[h] = mine < a.cols ? 4 + (uint32_t)(mine % a.block) / 2 : 4;
    }
    uint32_t scale_at[H], word_at[H];                             // of the lane's first row, from the block's (rows 24 apart: below 2^32)
#pragma unroll
    for (int h = 0; h < H; ++h) {
        scale_at[h] = 8 * j * (uint32_t)a.row_bytes;
        word_at[h] = scale_at[h] + at[h];
    }
    auto fetch_row = [&](R& v, uint32_t b, int e) {               // row e of the lane's eight; all 256 rows are there
        const uint64_t r0 = r_begin + (uint64_t)b * kBlockRows + wave * kStep;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            uint32_t of_scale = scale_at[h], of_word = word_at[h];
            asm volatile("" : "+v"(of_scale), "+v"(of_word));     // 32 bits here, too: the loads add them to a scalar base
            const uint8_t* p = block[h] + (r0 + e) * a.row_bytes;
            v.scale[h][e] = *reinterpret_cast<const float*>(p + of_scale);
            v.w[h][e] = *reinterpret_cast<const uint32_t*>(p + of_word);
        }
    };
    auto fetch_tail = [&](R& v, uint32_t b) {                     // rows behind the last repeat it (dy is 0 there)
        const uint64_t r0 = r_begin + (uint64_t)b * kBlockRows + wave * kStep + 8 * j;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint64_t row = r0 + e < a.rows ? r0 + e : a.rows - 1;
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const uint8_t* p = block[h] + row * a.row_bytes;
                v.scale[h][e] = *reinterpret_cast<const float*>(p);
                v.w[h][e] = *reinterpret_cast<const uint32_t*>(p + at[h]);
            }
        }
    };
    const T* dy_at[PIECES];                                       // of the thread's pieces, in row 0
#pragma unroll
    for (uint32_t q = 0; q < PIECES; ++q) {
        const uint32_t piece = q * kThreads + threadIdx.x, tok = piece / PER < tokens ? piece / PER : tokens - 1;
        dy_at[q] = static_cast<const T*>(a.in) + tok * a.in_ld + piece % PER * E;
    }
    auto fetch_dy = [&](Piece& v, uint32_t q, uint32_t b) { v = *reinterpret_cast<const Piece*>(dy_at[q] + (r_begin + (uint64_t)b * kBlockRows)); };
    auto fetch_dy_tail = [&](Piece (&v)[PIECES], uint32_t b) {
        const uint64_t r0 = r_begin + (uint64_t)b * kBlockRows;
#pragma unroll
        for (uint32_t q = 0; q < PIECES; ++q) {
            const uint64_t r = r0 + (q * kThreads + threadIdx.x) % PER * E;
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) v[q][e] = r + e < a.rows ? dy_at[q][r0 + e] : (T)0.f;
        }
    };
    auto stage_dy = [&](const Piece (&v)[PIECES], uint32_t buffer) {
#pragma unroll
        for (uint32_t q = 0; q < PIECES; ++q) {
            const uint32_t piece = q * kThreads + threadIdx.x;
            *reinterpret_cast<u32x4*>(staged + (buffer * TT * 16 + piece / PER) * kPitch + piece % PER * E) = __builtin_bit_cast(u32x4, v[q]);
        }
    };

    f32x4 sum[TT][8], off[TT][H];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < H; ++h) off[t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const CodeMasks masks = code_masks<__bf16>();
    auto use = [&](const R& v, uint32_t buffer, bool ragged, uint64_t r0, auto meanwhile) {   // meanwhile(c), c = 0 .. 7: next to a column's products
#pragma unroll
        for (int h = 0; h < H; ++h) {
            constexpr int COLS = NARROW ? 4 : 8;
            float unit[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) unit[e] = v.scale[h][e] * kPerCode;
            Eight<__bf16> left[TT][P];
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const T* from = staged + (buffer * TT * 16 + 16 * t + n) * kPitch + wave * kStep + 8 * j;
                const Eights raw = *reinterpret_cast<const Eights*>(from);
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = (float)raw[e] * unit[e];
                if (ragged)                                       // (a scale of the last row may be infinite)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] = r0 + 8 * j + e < a.rows ? d[e] : 0.f;
                split_operand<P>(d, left[t]);
            }
            f32x4 centre[TT];                                     // what codes are too large by
#pragma unroll
            for (int t = 0; t < TT; ++t) centre[t] = kCentred ? f32x4{0.f, 0.f, 0.f, 0.f} : off[t][h];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int t = 0; t < TT; ++t) centre[t] = matrix_fma(left[t][p], centre_operand<__bf16>(), centre[t]);
            if (!kCentred)
#pragma unroll
                for (int t = 0; t < TT; ++t) off[t][h] = centre[t];
#pragma unroll
            for (int g = 0; g < COLS / 4; ++g) {
                uint32_t pair[4];                                 // four columns of rows 2 q and 2 q + 1
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t select = NARROW ? (n % 2 ? 0x07060302u : 0x05040100u) : g ? 0x07060302u : 0x05040100u;
                    pair[q] = __builtin_amdgcn_perm(v.w[h][2 * q + 1], v.w[h][2 * q], select);
                }
                auto column = [&](auto which) {
                    constexpr int N = decltype(which)::value;
                    const int c = COLS * h + 4 * g + N;
                    const u32x4 codes = {code_pair<__bf16, N>(pair[0], masks), code_pair<__bf16, N>(pair[1], masks), code_pair<__bf16, N>(pair[2], masks),
                                         code_pair<__bf16, N>(pair[3], masks)};
                    const Eight<__bf16> right = __builtin_bit_cast(Eight<__bf16>, codes);
                    meanwhile(c);
                    f32x4 part[TT];
#pragma unroll
                    for (int t = 0; t < TT; ++t) part[t] = kCentred ? -centre[t] : sum[t][c];
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int t = 0; t < TT; ++t) part[t] = matrix_fma(left[t][p], right, part[t]);
#pragma unroll
                    for (int t = 0; t < TT; ++t) sum[t][c] = kCentred ? sum[t][c] + part[t] : part[t];
                    __builtin_amdgcn_sched_barrier(0);
                };
                column(std::integral_constant<int, 0>());
                column(std::integral_constant<int, 1>());
                column(std::integral_constant<int, 2>());
                column(std::integral_constant<int, 3>());
            }
        }
    };
    // Whole blocks of rows.  While one is multiplied the next one's codes are read, two rows next to each of the first columns' products, and the dy of the one
    // after that, next to the others'; dy of the next one goes into LDS.  (Behind the end the last one is read again: no branch, so that loads can be counted.)
    const uint32_t whole = (uint32_t)((r_end - r_begin) / kBlockRows);
    Piece dy[PIECES];
    if (whole) {
        R rows[2];
        auto within = [&](uint32_t b) { return b < whole ? b : whole - 1; };
#pragma unroll
        for (uint32_t q = 0; q < PIECES; ++q) fetch_dy(dy[q], q, 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) fetch_row(rows[0], 0, e);
        stage_dy(dy, 0);
#pragma unroll
        for (uint32_t q = 0; q < PIECES; ++q) fetch_dy(dy[q], q, within(1));
        __syncthreads();
        auto step = [&](const R& now, R& next, uint32_t b) {
            use(now, b & 1, false, 0, [&](int c) {
                if (c == 0) stage_dy(dy, (b + 1) & 1);
                if (c < 4) {
                    fetch_row(next, within(b + 1), 2 * c);
                    fetch_row(next, within(b + 1), 2 * c + 1);
#pragma unroll
                    for (uint32_t q = c; q < PIECES; q += 4) fetch_dy(dy[q], q, within(b + 2));
                }
            });
            __syncthreads();
        };
        for (uint32_t b = 0; b < whole; b += 2) {
            step(rows[0], rows[1], b);
            if (b + 1 >= whole) break;
            step(rows[1], rows[0], b + 1);
        }
    }
    if (whole < blocks) {                                         // ... and the rows that are left
        R rows;
        fetch_dy_tail(dy, whole);
        fetch_tail(rows, whole);
        stage_dy(dy, 0);
        __syncthreads();
        const uint64_t r0 = r_begin + (uint64_t)whole * kBlockRows + wave * kStep;
        use(rows, 0, true, r0, [](int) {});
        __syncthreads();
    }
    if constexpr (!kCentred)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[t][c] -= off[t][NARROW ? c / 4 : 0];

    // join the waves, CT columns of each word at a time: [wave][column][token tile][lane], then rows of 128 columns
    constexpr int CT = 8 / TT;
    f32x4* joined = reinterpret_cast<f32x4*>(lds);
    float* line = reinterpret_cast<float*>(lds + kWaves * CT * TT * 64 * sizeof(f32x4));       // [token][128 + 4]
#pragma unroll
    for (int c0 = 0; c0 < 8; c0 += CT) {
        if (c0) __syncthreads();
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int t = 0; t < TT; ++t) joined[((wave * CT + c) * TT + t) * 64 + lane] = sum[t][c0 + c];
        __syncthreads();
        for (uint32_t q = wave; q < CT * TT; q += kWaves) {
            const uint32_t c = c0 + q / TT, t = q % TT;
            f32x4 s = joined[q * 64 + lane];
            for (int w = 1; w < kWaves; ++w) s += joined[(w * CT * TT + q) * 64 + lane];
            const uint32_t col = NARROW ? c / 4 * 64 + 4 * n + c % 4 : 8 * n + c;
#pragma unroll
            for (int i = 0; i < 4; ++i) line[(16 * t + 4 * j + i) * (kChunk + 4) + col] = s[i];
        }
    }
    __syncthreads();
    for (uint32_t q = threadIdx.x; q < tokens * kChunk; q += kThreads) {
        const uint32_t tok = q / kChunk, c = q % kChunk;
        if (col0 + c >= a.cols) continue;
        const float v = line[tok * (kChunk + 4) + c];
        if (a.partial) a.partial[(part * tokens + tok) * a.cols + col0 + c] = v;
        else gradient_store<T>(a, col0 + c, tok, v);
    }
}

// Adds the parts.  A thread per column and token.
template <typename T>
__global__ void __launch_bounds__(256) product_gradient_join_kernel(GradientShape a) {
    const uint64_t c = (a.chunk0 * (uint64_t)gridDim.x + blockIdx.x) * 256 + threadIdx.x, t = blockIdx.y;
    if (c >= a.cols) return;
    const float* from = a.partial + t * a.cols + c;
    const uint64_t step = a.tokens * a.cols;
    float v = 0.f;
    for (uint32_t p = 0; p < a.parts; p += 8) {
        float w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = p + q < a.parts ? from[(p + q) * step] : 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) v += w[q];
    }
    gradient_store<T>(a, c, t, v);
}

// Workgroups split the rows until all compute units have one, and not one more, which would take as long again; where two fit into a unit's registers, two.
// 32768 x 4096, bf16, blocks of 256, us, for 256 : 512 workgroups: 64 tokens 46.1 : 54.4 (33 columns of them, 231 : 495, 49.8 : 55.5; 264 took 82), 32 tokens
// 28.7 : 32.6; 16 tokens 22.0 : 20.2; 16 tokens of 8192 x 5000, fp32, 14.7 : 14.6 (320: 17.9).
void gradient_plan(uint64_t rows, uint64_t cols, uint64_t tokens, bool narrow, uint32_t& parts, uint64_t& part_rows) {
    const uint64_t chunks = (cols + kChunk - 1) / kChunk, blocks = (rows + kBlockRows - 1) / kBlockRows;
    uint64_t p = (tokens <= 16 && !narrow ? 512 : 256) / chunks;
    if (p > blocks) p = blocks;
    if (p > 64) p = 64;
    if (!p || blocks <= 4) p = 1;                                 // (7 x 1024 x 2000, bf16: 1 part 8.4 us, 4: 5.6 and 2.6 of the launch that joins them; 512 rows 6.4, and 7.8)
    const uint64_t each = (blocks + p - 1) / p;
    part_rows = each * kBlockRows;
    parts = (uint32_t)((blocks + each - 1) / each);
}

template <typename T, int TT, bool NARROW>
void launch_gradient_kernel(const GradientShape& a, hipStream_t stream) {
    constexpr uint32_t join = kWaves * 8 * 64 * 16 + 16 * TT * (kChunk + 4) * 4, stage = 2 * TT * 16 * (kBlockRows * sizeof(T) + 16);
    constexpr uint32_t bytes = join > stage ? join : stage;
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(product_gradient_kernel<T, TT, NARROW>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    GradientShape b = a;
    for (uint64_t g = 0; g < a.chunks; g += kGroupsOfLaunch) {
        b.chunk0 = g;
        const uint64_t here = a.chunks - g < kGroupsOfLaunch ? a.chunks - g : kGroupsOfLaunch;
        hipLaunchKernelGGL((product_gradient_kernel<T, TT, NARROW>), dim3((unsigned)here, a.parts), dim3(kThreads), bytes, stream, b);
    }
}

template <typename T>
void launch_gradient_of(const ProductArgs& args, hipStream_t stream) {
    const bool narrow = args.block == 64;
    const uint64_t most = kTokens<T>(narrow);
    for (uint64_t t0 = 0; t0 < args.tokens; t0 += most) {
        GradientShape a{};
        static_cast<ProductArgs&>(a) = args;
        a.tokens = args.tokens - t0 < most ? args.tokens - t0 : most;
        a.in = static_cast<const T*>(args.in) + t0 * args.in_ld;
        a.out = static_cast<T*>(args.out) + t0 * args.out_ld;
        a.chunks = (a.cols + kChunk - 1) / kChunk;
        gradient_plan(a.rows, a.cols, a.tokens, narrow, a.parts, a.part_rows);
        a.partial = a.parts > 1 ? static_cast<float*>(a.work) : nullptr;
        if (a.tokens <= 16) narrow ? launch_gradient_kernel<T, 1, true>(a, stream) : launch_gradient_kernel<T, 1, false>(a, stream);
        else if (a.tokens <= 32) narrow ? launch_gradient_kernel<T, 2, true>(a, stream) : launch_gradient_kernel<T, 2, false>(a, stream);
        else if constexpr (kTokens<T>(false) > 32) launch_gradient_kernel<T, 4, false>(a, stream);
        if (!a.partial) continue;
        a.chunk0 = 0;                                             // (parts are only for matrices of at most 256 chunks)
        hipLaunchKernelGGL(product_gradient_join_kernel<T>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)a.tokens), dim3(256), 0, stream, a);
    }
}

}  // namespace

uint64_t product_gradient_work_bytes(const ds_matrix& m) {
    const bool narrow = m.block == 64;
    uint64_t most = 0, bytes = 0;
    by_dtype(m.dtype, [&](auto kind) { most = kTokens<decltype(kind)>(narrow); });
    for (uint64_t tokens : {m.tokens < most ? m.tokens : most, m.tokens % most}) {             // of the launches: whole ones and the last
        uint32_t parts;
        uint64_t part_rows;
        gradient_plan(m.rows, m.cols, tokens, narrow, parts, part_rows);
        const uint64_t here = parts > 1 ? parts * tokens * m.cols * sizeof(float) : 0;
        if (here > bytes) bytes = here;
    }
    return bytes;
}

hipError_t launch_product_gradient(const ProductArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_gradient_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
