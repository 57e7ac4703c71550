// The norms of gradients that lie in many tensors, and clipping (ds_gradients_lay, ds_gradient_norm, ds_clip).
//
// Work goes by tiles of 16384 elements, a workgroup each; a table that is laid once says which tensor a tile is of.  The sum of squares of a tile goes to
// work_dev, a workgroup per worker adds them up in an order that is always the same, and for clipping a last launch reads the tensors once more, from the last
// tile to the first: what the sums read last is what the memory-side cache still holds.
//   Squares and sums are in 64 bits: 32 would overflow from 1.8e19 on and lose what is below 1e-23, and a 64-bit multiply-add takes no longer than one of 32.
#include "dsq_answers.h"

namespace dsq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint64_t kTilesOfLaunch = 1u << 22;                     // a launch dimension holds fewer than 2^32 work-items

struct Table {
    const TensorRecord* record;
    const uint64_t* first_tile;
    const uint32_t* tensor_of;
};
__host__ __device__ inline Table table_of(const ds_gradients& g) {
    Table t;
    t.record = static_cast<const TensorRecord*>(g.table_dev);
    t.first_tile = reinterpret_cast<const uint64_t*>(t.record + g.tensors + 1);
    t.tensor_of = reinterpret_cast<const uint32_t*>(t.first_tile + g.workers + 1);
    return t;
}

// A workgroup per record: itself, the first tile of the workers that begin with it, and its tiles' owner.
__global__ void __launch_bounds__(kThreads) lay_kernel(ds_gradients g, RecordBatch batch) {
    const Table t = table_of(g);
    const TensorRecord r = batch.record[blockIdx.x];
    const uint64_t at = batch.first + blockIdx.x;
    if (threadIdx.x == 0) const_cast<TensorRecord*>(t.record)[at] = r;
    for (uint64_t w = r.worker_from + threadIdx.x; w <= r.worker; w += kThreads) const_cast<uint64_t*>(t.first_tile)[w] = r.first_tile;
    const uint64_t tiles = (r.count + kGradientTile - 1) / kGradientTile;
    for (uint64_t i = threadIdx.x; i < tiles; i += kThreads) const_cast<uint32_t*>(t.tensor_of)[r.first_tile + i] = (uint32_t)at;
}

template <typename F>
__device__ __forceinline__ void of_dtype(uint32_t dtype, F f) {
    if (dtype == DS_BF16) f(__bf16());
    else if (dtype == DS_F16) f(_Float16());
    else f(float());
}

// 16 bytes of elements, at any element's address.
template <typename T>
struct Elements {
    static constexpr uint32_t E = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    static constexpr uint32_t kPieces = kGradientTile / (kThreads * E);
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// Over the workgroup, in every thread.  sums: WAVES doubles of LDS, not read by anybody any more.
template <int WAVES>
__device__ __forceinline__ double workgroup_sum(double v, double* sums) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = v;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all += sums[w];
    return all;
}

// The part of a tile that the thread has: kPieces pieces, thread after thread, and of a tile with an odd end an element more.
template <typename T>
struct Tile {
    using Piece = typename Elements<T>::Piece;
    static constexpr uint32_t E = Elements<T>::E, kPieces = Elements<T>::kPieces;
    Piece piece[kPieces];
    T last;
    uint32_t whole;                                               // pieces of the tile
    uint32_t n;

    __device__ __forceinline__ Tile(const T* from, uint32_t n) : last((T)0.f), whole(n / E), n(n) {
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) {
            const uint32_t at = p * kThreads + threadIdx.x;
            if (at < whole) piece[p] = *reinterpret_cast<const Piece*>(from + at * E);
            else
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) piece[p][e] = (T)0.f;
        }
        if (has_last()) last = from[whole * E + threadIdx.x];
    }
    __device__ __forceinline__ bool has_last() const { return whole * E + threadIdx.x < n; }
    __device__ __forceinline__ double squares() const {
        double sum[2] = {(double)(float)last * (double)(float)last, 0.0};
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p)
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) {
                const double x = (double)(float)piece[p][e];
                sum[e & 1] = fma(x, x, sum[e & 1]);
            }
        return sum[0] + sum[1];
    }
    // Writes factor times it; zeros for a factor of 0.
    template <typename O>
    __device__ __forceinline__ void write(O* to, double factor) const {
        auto scaled = [&](T x) { return factor == 0.0 ? (O)0.f : (O)(float)((double)(float)x * factor); };
        constexpr uint32_t M = 16 / sizeof(O) < E ? 16 / sizeof(O) : E;                    // elements of a store
        typedef O Out __attribute__((ext_vector_type(M), aligned(sizeof(O))));
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) {
            const uint32_t at = p * kThreads + threadIdx.x;
            if (at >= whole) break;
#pragma unroll
            for (uint32_t s = 0; s < E; s += M) {
                Out out;
#pragma unroll
                for (uint32_t e = 0; e < M; ++e) out[e] = scaled(piece[p][s + e]);
                *reinterpret_cast<Out*>(to + at * E + s) = out;
            }
        }
        if (has_last()) to[whole * E + threadIdx.x] = scaled(last);
    }
};

struct TileOf {
    const TensorRecord& r;
    uint64_t from;                                                // elements of the tensor before it
    uint32_t n;
    __device__ __forceinline__ TileOf(const Table& t, uint64_t tile) : r(t.record[t.tensor_of[tile]]) {
        from = (tile - r.first_tile) * kGradientTile;
        n = r.count - from < kGradientTile ? (uint32_t)(r.count - from) : kGradientTile;
    }
};

struct ClipShape : ClipArgs {
    double* squares;                                              // [tile]
    double* factor;                                               // [worker]
    uint64_t tile0;
};

__global__ void __launch_bounds__(kThreads) squares_kernel(ClipShape a) {
    __shared__ double sums[kWaves];
    const uint64_t tile = a.tile0 + blockIdx.x;
    const TileOf t(table_of(a.g), tile);
    double mine = 0.0;
    of_dtype(t.r.dtype, [&](auto kind) {
        using T = decltype(kind);
        mine = Tile<T>(static_cast<const T*>(t.r.data) + t.from, t.n).squares();
    });
    const double all = workgroup_sum<kWaves>(mine, sums);
    if (threadIdx.x == 0) a.squares[tile] = all;
}

__device__ __forceinline__ double factor_of(double norm, double max_norm) {
    if (!(norm < __builtin_huge_val())) return 0.0;
    return norm > max_norm ? max_norm / norm : 1.0;
}

constexpr int kJoinThreads = 1024;
__global__ void __launch_bounds__(kJoinThreads) norm_kernel(ClipShape a) {
    __shared__ double sums[kJoinThreads / 64];
    const Table t = table_of(a.g);
    const uint64_t end = t.first_tile[blockIdx.x + 1];
    double mine = 0.0;
    for (uint64_t i = t.first_tile[blockIdx.x] + threadIdx.x; i < end; i += kJoinThreads) mine += a.squares[i];
    const double norm = sqrt(workgroup_sum<kJoinThreads / 64>(mine, sums));
    if (threadIdx.x != 0) return;
    if (a.norm) a.norm[blockIdx.x] = (float)norm;
    if (a.factor) a.factor[blockIdx.x] = factor_of(norm, a.max_norm);
}

__global__ void __launch_bounds__(kThreads) scale_kernel(ClipShape a) {
    const uint64_t tile = a.g.tiles - 1 - (a.tile0 + blockIdx.x);
    const TileOf t(table_of(a.g), tile);
    const double factor = a.factor[t.r.worker];
    if (!a.out && factor == 1.0) return;
    of_dtype(t.r.dtype, [&](auto kind) {
        using T = decltype(kind);
        T* data = static_cast<T*>(t.r.data) + t.from;
        const Tile<T> mine(data, t.n);
        if (a.out) mine.write(a.out + t.r.worker * a.out_ld + t.r.column + t.from, factor);
        else mine.write(data, factor);
    });
}

template <typename F>
void over_tiles(ClipShape& a, F launch) {
    for (a.tile0 = 0; a.tile0 < a.g.tiles; a.tile0 += kTilesOfLaunch)
        launch(dim3((unsigned)(a.g.tiles - a.tile0 < kTilesOfLaunch ? a.g.tiles - a.tile0 : kTilesOfLaunch)));
}

ClipShape shape_of(const ClipArgs& args, bool scale) {
    ClipShape a{};
    static_cast<ClipArgs&>(a) = args;
    a.squares = static_cast<double*>(a.work);
    a.factor = scale ? a.squares + a.g.tiles : nullptr;
    return a;
}

void launch_norms(ClipShape& a, hipStream_t stream) {
    over_tiles(a, [&](dim3 grid) { hipLaunchKernelGGL(squares_kernel, grid, dim3(kThreads), 0, stream, a); });
    hipLaunchKernelGGL(norm_kernel, dim3((unsigned)a.g.workers), dim3(kJoinThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_lay(const ds_gradients& g, const RecordBatch& batch, hipStream_t stream) {
    hipLaunchKernelGGL(lay_kernel, dim3((unsigned)batch.here), dim3(kThreads), 0, stream, g, batch);
    return hipGetLastError();
}

uint64_t gradient_norm_work_bytes(const ds_gradients& g) { return g.tiles * sizeof(double); }

hipError_t launch_gradient_norm(const ClipArgs& args, hipStream_t stream) {
    ClipShape a = shape_of(args, false);
    launch_norms(a, stream);
    return hipGetLastError();
}

uint64_t clip_work_bytes(const ds_gradients& g) { return (g.tiles + g.workers) * sizeof(double); }

hipError_t launch_clip(const ClipArgs& args, hipStream_t stream) {
    ClipShape a = shape_of(args, true);
    launch_norms(a, stream);
    over_tiles(a, [&](dim3 grid) { hipLaunchKernelGGL(scale_kernel, grid, dim3(kThreads), 0, stream, a); });
    return hipGetLastError();
}

}  // namespace dsq
