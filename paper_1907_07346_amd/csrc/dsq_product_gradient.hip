// The gradient of ds_product with respect to its vectors (ds_product_gradient): dx = dy M, M's rows as 4-bit codes with a scale per block.
//
// The sum runs over the matrix's rows, so the scales belong to what is summed: dy * scale is the other operand, made anew for every block
// of columns and rounded to bf16 pieces (two for 16-bit dtypes, 2^-17 relative, three for fp32: 24 bits).  A wave takes 128 columns and 32
// rows at a time: lane (n, j) loads word n (eight columns) of rows 8 j .. 8 j + 7, and column c of all words, c = 0 .. 7, is one matrix
// instruction: codes of two rows sit in the halves of a register after one byte permutation, two more instructions make operands of two (dsq_codes.h).
// The waves of a workgroup and the workgroups of a column take different rows; the waves join in LDS, the workgroups through fp32 partial sums in
// work_dev and a second launch.
#include "dsq_answers.h"
#include "dsq_codes.h"

namespace dsq {
namespace {

constexpr int kWaves = 8, kChunk = 128, kStep = 32;               // waves of a workgroup; columns and rows a wave takes at a time
constexpr uint64_t kTokens = 64;                                  // of a launch
constexpr uint64_t kGroupsOfLaunch = 1u << 22;                    // a launch dimension holds fewer than 2^32 work-items

struct GradientShape : ProductArgs {
    uint32_t parts;                                               // workgroups that split the rows
    uint64_t part_rows;                                           // a multiple of kStep
    uint64_t chunks, chunk0;
    float* partial;                                               // parts x tokens x cols, or nullptr
};

// One weight after the other, as the formula has it: for a result that is not finite.
template <typename T>
__device__ __noinline__ float gradient_in_order(const ProductArgs& a, uint64_t c, uint64_t t) {
    const uint8_t* block = a.msg + c / a.block * (4 + a.block / 2);
    const uint32_t at = c % a.block / 8, by = c % 8 * 4;
    const T* dy = static_cast<const T*>(a.in) + t * a.in_ld;
    float sum = 0.f;
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

// What a wave needs of 32 rows.  A matrix instruction's columns must share a block: with blocks of 64 a lane takes four columns of either
// block, half of word n / 2, and its column c is 64 floor(c / 4) + 4 n + c % 4 instead of 8 n + c.
template <typename T, int TT, bool NARROW>
struct Rows {
    static constexpr int H = NARROW ? 2 : 1;
    uint32_t w[H][8];
    float scale[H][8];
    typedef T Eights __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    Eights dy[TT];
};

template <typename T, int TT, bool NARROW>
__global__ void __launch_bounds__(kWaves * 64, 2) product_gradient_kernel(GradientShape a) {
    constexpr int P = sizeof(T) == 4 ? 3 : 2, H = NARROW ? 2 : 1;
    using R = Rows<T, TT, NARROW>;
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, n = lane & 15, j = lane >> 4;
    const uint32_t tokens = (uint32_t)a.tokens;
    // Workgroups go round the eight XCDs: those of the same rows, which share cache lines, onto one of them.
    uint64_t chunk = blockIdx.x, part = blockIdx.y;
    if (a.parts % 8 == 0) {
        const uint64_t id = (uint64_t)blockIdx.y * gridDim.x + blockIdx.x, q = id / 8;
        part = id % 8 + q / gridDim.x * 8;
        chunk = q % gridDim.x;
    }
    const uint64_t col0 = (a.chunk0 + chunk) * kChunk;
    const uint64_t r_end = (part + 1) * a.part_rows < a.rows ? (part + 1) * a.part_rows : a.rows;

    const uint32_t pitch = 4 + a.block / 2;
    const uint8_t* block[H];                                      // in row 0: the blocks, and the lane's word in them
    uint32_t at[H];
    bool there[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const uint64_t col = col0 + 64 * h, mine = NARROW ? col + n / 2 * 8 : col + 8 * n;
        block[h] = a.msg + (col < a.cols ? col : 0) / a.block * pitch;
        there[h] = mine < a.cols;
        at[h] = there[h] ? 4 + (uint32_t)(mine % a.block) / 2 : 4;
    }
    auto load = [&](R& v, uint64_t r0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint64_t r = r0 + 8 * j + e, row = r < a.rows ? r : a.rows - 1;      // rows behind the last: dy counts as 0 there
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const uint8_t* p = block[h] + row * a.row_bytes;
                v.scale[h][e] = *reinterpret_cast<const float*>(p);
                v.w[h][e] = *reinterpret_cast<const uint32_t*>(p + at[h]);
            }
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const uint32_t tok = 16 * t + n < tokens ? 16 * t + n : tokens - 1;
            const T* dy = static_cast<const T*>(a.in) + tok * a.in_ld + r0 + 8 * j;
            if (r0 + kStep <= a.rows) v.dy[t] = *reinterpret_cast<const typename R::Eights*>(dy);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v.dy[t][e] = r0 + 8 * j + e < a.rows ? dy[e] : (T)0.f;
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
    auto use = [&](const R& v, uint64_t r0) {
        const bool ragged = r0 + kStep > a.rows;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            Eight<__bf16> left[TT][P];
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[e] = (float)v.dy[t][e] * (v.scale[h][e] * kPerCode);
                    if (ragged && r0 + 8 * j + e >= a.rows) d[e] = 0.f;
                }
                split_operand<__bf16, P>(d, left[t]);
#pragma unroll
                for (int p = 0; p < P; ++p) off[t][h] = matrix_fma(left[t][p], centre_operand<__bf16>(), off[t][h]);
            }
            uint32_t pair[H == 2 ? 1 : 2][4];                     // columns 0 .. 3 (and 4 .. 7) of rows 2 q and 2 q + 1
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (NARROW) {
                    pair[0][q] = __builtin_amdgcn_perm(v.w[h][2 * q + 1], v.w[h][2 * q], n % 2 ? 0x07060302u : 0x05040100u);
                } else {
                    pair[0][q] = __builtin_amdgcn_perm(v.w[0][2 * q + 1], v.w[0][2 * q], 0x05040100u);
                    pair[1][q] = __builtin_amdgcn_perm(v.w[0][2 * q + 1], v.w[0][2 * q], 0x07060302u);
                }
            }
            auto column = [&](auto which, int g) {                // column `which` of the four, of pair[g]
                constexpr int N = decltype(which)::value;
                const u32x4 codes = {code_pair<__bf16, N>(pair[g][0]), code_pair<__bf16, N>(pair[g][1]), code_pair<__bf16, N>(pair[g][2]),
                                     code_pair<__bf16, N>(pair[g][3])};
                const Eight<__bf16> right = __builtin_bit_cast(Eight<__bf16>, codes);
                const int c = (NARROW ? 4 * h : 4 * g) + N;
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int p = 0; p < P; ++p) sum[t][c] = matrix_fma(left[t][p], right, sum[t][c]);
            };
#pragma unroll
            for (int g = 0; g < (NARROW ? 1 : 2); ++g) {
                column(std::integral_constant<int, 0>(), g);
                column(std::integral_constant<int, 1>(), g);
                column(std::integral_constant<int, 2>(), g);
                column(std::integral_constant<int, 3>(), g);
            }
        }
    };
    uint64_t r0 = part * a.part_rows + wave * kStep;
    R next;
    if (r0 < r_end) load(next, r0);
    for (; r0 < r_end; r0 += kWaves * kStep) {
        const R now = next;
        if (r0 + kWaves * kStep < r_end) load(next, r0 + kWaves * kStep);
        use(now, r0);
    }
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
    for (uint32_t q = threadIdx.x; q < tokens * kChunk; q += kWaves * 64) {
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
    float v = 0.f;
    for (uint32_t p = 0; p < a.parts; ++p) v += a.partial[(p * a.tokens + t) * a.cols + c];
    gradient_store<T>(a, c, t, v);
}

void gradient_plan(uint64_t rows, uint64_t cols, uint32_t& parts, uint64_t& part_rows) {
    const uint64_t chunks = (cols + kChunk - 1) / kChunk, steps = (rows + kStep - 1) / kStep;
    uint64_t p = 1;
    while (chunks * p < 256 && steps >= 2 * p * kWaves && p < 64) p *= 2;
    const uint64_t each = (steps + p - 1) / p;
    part_rows = each * kStep;
    parts = (uint32_t)((steps + each - 1) / each);
}

template <typename T, int TT, bool NARROW>
void launch_gradient_kernel(const GradientShape& a, hipStream_t stream) {
    constexpr uint32_t bytes = kWaves * 8 * 64 * 16 + 16 * TT * (kChunk + 4) * 4;
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(product_gradient_kernel<T, TT, NARROW>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    GradientShape b = a;
    for (uint64_t g = 0; g < a.chunks; g += kGroupsOfLaunch) {
        b.chunk0 = g;
        const uint64_t here = a.chunks - g < kGroupsOfLaunch ? a.chunks - g : kGroupsOfLaunch;
        hipLaunchKernelGGL((product_gradient_kernel<T, TT, NARROW>), dim3((unsigned)here, a.parts), dim3(kWaves * 64), bytes, stream, b);
    }
}

template <typename T>
void launch_gradient_of(const ProductArgs& args, hipStream_t stream) {
    for (uint64_t t0 = 0; t0 < args.tokens; t0 += kTokens) {
        GradientShape a{};
        static_cast<ProductArgs&>(a) = args;
        a.tokens = args.tokens - t0 < kTokens ? args.tokens - t0 : kTokens;
        a.in = static_cast<const T*>(args.in) + t0 * args.in_ld;
        a.out = static_cast<T*>(args.out) + t0 * args.out_ld;
        a.chunks = (a.cols + kChunk - 1) / kChunk;
        gradient_plan(a.rows, a.cols, a.parts, a.part_rows);
        a.partial = a.parts > 1 ? static_cast<float*>(a.work) : nullptr;
        const bool narrow = a.block == 64;
        if (a.tokens <= 16) narrow ? launch_gradient_kernel<T, 1, true>(a, stream) : launch_gradient_kernel<T, 1, false>(a, stream);
        else if (a.tokens <= 32) narrow ? launch_gradient_kernel<T, 2, true>(a, stream) : launch_gradient_kernel<T, 2, false>(a, stream);
        else narrow ? launch_gradient_kernel<T, 4, true>(a, stream) : launch_gradient_kernel<T, 4, false>(a, stream);
        if (!a.partial) continue;
        a.chunk0 = 0;                                             // (parts are only for matrices of fewer than 256 chunks)
        hipLaunchKernelGGL(product_gradient_join_kernel<T>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)a.tokens), dim3(256), 0, stream, a);
    }
}

}  // namespace

uint64_t product_gradient_work_bytes(const ds_matrix& m) {
    uint32_t parts;
    uint64_t part_rows;
    gradient_plan(m.rows, m.cols, parts, part_rows);
    return parts > 1 ? (uint64_t)parts * (m.tokens < kTokens ? m.tokens : kTokens) * m.cols * sizeof(float) : 0;
}

hipError_t launch_product_gradient(const ProductArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) { launch_gradient_of<decltype(kind)>(a, stream); });
    return hipGetLastError();
}

}  // namespace dsq
