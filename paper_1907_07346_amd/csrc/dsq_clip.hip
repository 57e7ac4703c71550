// The norms of gradients that lie in many tensors, and clipping (ds_gradients_lay, ds_gradient_norm, ds_clip).
//
// Work goes by tiles of 16384 elements, a workgroup each; a table that is laid once says which tensor a tile is of.  The sum of squares of a tile goes to
// work_dev, a workgroup per worker adds them up in an order that is always the same, and for clipping a last launch reads the tensors once more, from the last
// tile to the first: what the sums read last is what the memory-side cache still holds.
//   Squares and sums are in 64 bits: 32 would overflow from 1.8e19 on and lose what is below 1e-23, and a 64-bit multiply-add takes no longer than one of 32.
//   Memory bounds both.  Norms of 8 x 25.6 million, bf16, in 161 tensors each: 65 us, 6.3 TB/s (a large copy: 6.6).  Clipping 32 x 25.6 million, fp32, into rows: 1650 us, of which the squares
// take 475 (6.9 TB/s) and the scaling 1170 (5.6, in and out).  It has to read twice, as a factor depends on the last element and no cache holds the first; 16 x 11.2 million, mixed, 256 us.  In
// place: 32 x 25.6 million, fp32, 1690 us, 8 x 25.6 million, bf16, 222; where nothing is above the limit 960 and 136, twice the norm's 478 and 73, as the tiles are asked for before the factor is known.
#include <type_traits>

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

// The squares of the thread's part of a tile: kPieces pieces, thread after thread, and of a tile with an odd end an element more.
template <bool ONCE, typename T>
__device__ __forceinline__ double squares(const T* from, uint32_t n) {
    using Piece = typename Elements<T>::Piece;
    constexpr uint32_t E = Elements<T>::E, kPieces = Elements<T>::kPieces;
    const uint32_t whole = n / E;
    Piece piece[kPieces];
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) {
        const uint32_t at = p * kThreads + threadIdx.x;
        const Piece* const place = reinterpret_cast<const Piece*>(from + at * E);
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) piece[p][e] = (T)0.f;
        if (at < whole) piece[p] = ONCE ? __builtin_nontemporal_load(place) : *place;
    }
    const double last = whole * E + threadIdx.x < n ? (double)(float)from[whole * E + threadIdx.x] : 0.0;
    double sum[2] = {last * last, 0.0};
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p)
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) {
            const double x = (double)(float)piece[p][e];
            sum[e & 1] = fma(x, x, sum[e & 1]);
        }
    return sum[0] + sum[1];
}

// Writes factor() times a tile, zeros for a factor of 0 and nothing for one of 1 if it would change nothing.  Four elements at a time, so that a wave's stores of fp32 are whole lines
// one behind the other, from the first place on at which they are; the tile is on its way while the factor is made.
template <bool ONCE, typename T, typename O, typename F>
__device__ __forceinline__ void scale(const T* from, O* to, uint32_t n, F factor_of_worker) {
    typedef T In __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef O Out __attribute__((ext_vector_type(4)));
    constexpr uint32_t kFours = kGradientTile / (4 * kThreads), kLine = 128 / sizeof(O);
    uint32_t head = (kLine - (uint32_t)(reinterpret_cast<uintptr_t>(to) / sizeof(O)) % kLine) % kLine;
    if (head > n) head = n;
    const uint32_t fours = (n - head) / 4, tail = head + 4 * fours;                        // (n - tail < 4)
    In four[kFours];
#pragma unroll
    for (uint32_t p = 0; p < kFours; ++p) {
        const In* const place = reinterpret_cast<const In*>(from + head + (p * kThreads + threadIdx.x) * 4);
        if (p * kThreads + threadIdx.x < fours) four[p] = ONCE ? __builtin_nontemporal_load(place) : *place;
    }
    // a thread's element before the first line, or behind the last four
    const uint32_t odd = threadIdx.x < head ? threadIdx.x : tail + threadIdx.x - head;
    const float single = odd < n ? (float)from[odd] : 0.f;
    const double factor = factor_of_worker();
    if (std::is_same_v<T, O> && (const void*)from == (const void*)to && factor == 1.0) return;
    // (to 16 bits by way of fp32: 2^-25 of the value more than half a step)
    auto scaled = [&](T x) { return factor == 0.0 ? (O)0.f : (O)(float)((double)(float)x * factor); };
#pragma unroll
    for (uint32_t p = 0; p < kFours; ++p)
        if (p * kThreads + threadIdx.x < fours) {
            Out out;
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) out[e] = scaled(four[p][e]);
            Out* const at = reinterpret_cast<Out*>(to + head + (p * kThreads + threadIdx.x) * 4);
            if constexpr (ONCE) __builtin_nontemporal_store(out, at);
            else *at = out;
        }
    if (odd < n) to[odd] = factor == 0.0 ? (O)0.f : (O)(float)((double)single * factor);
}

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

template <bool ONCE>
__global__ void __launch_bounds__(kThreads) squares_kernel(ClipShape a) {
    __shared__ double sums[kWaves];
    const uint64_t tile = a.tile0 + blockIdx.x;
    const TileOf t(table_of(a.g), tile);
    double mine = 0.0;
    of_dtype(t.r.dtype, [&](auto kind) {
        using T = decltype(kind);
        mine = squares<ONCE>(static_cast<const T*>(t.r.data) + t.from, t.n);
    });
    const double all = workgroup_sum<kWaves>(mine, sums);
    if (threadIdx.x == 0) a.squares[tile] = all;
}

// The norm of a worker, out of its tiles' squares.
template <int THREADS>
__device__ __forceinline__ double norm_of(const ClipShape& a, uint64_t first, uint64_t end, double* sums) {
    double mine = 0.0;
    for (uint64_t i = first + threadIdx.x; i < end; i += THREADS) mine += a.squares[i];
    return sqrt(workgroup_sum<THREADS / 64>(mine, sums));
}
__device__ __forceinline__ double factor_of(double norm, double max_norm) {
    if (!(norm < __builtin_huge_val())) return 0.0;
    return norm > max_norm ? max_norm / norm : 1.0;
}

constexpr int kJoinThreads = 1024;
__global__ void __launch_bounds__(kJoinThreads) norm_kernel(ClipShape a) {
    __shared__ double sums[kJoinThreads / 64];
    const Table t = table_of(a.g);
    const double norm = norm_of<kJoinThreads>(a, t.first_tile[blockIdx.x], t.first_tile[blockIdx.x + 1], sums);
    if (threadIdx.x != 0) return;
    if (a.norm) a.norm[blockIdx.x] = (float)norm;
    if (a.factor) a.factor[blockIdx.x] = factor_of(norm, a.max_norm);
}

// JOINED: a launch has made the workers' factors; otherwise every workgroup makes its worker's, and that of a worker's first tile writes the norm.
template <bool ONCE, bool JOINED>
__global__ void __launch_bounds__(kThreads) scale_kernel(ClipShape a) {
    __shared__ double sums[kWaves];
    const uint64_t tile = a.g.tiles - 1 - (a.tile0 + blockIdx.x); // (the last first: it is the likeliest to be in a cache)
    const Table table = table_of(a.g);
    const TileOf t(table, tile);
    auto factor = [&] {
        if constexpr (JOINED) {
            return a.factor[t.r.worker];
        } else {
            const uint64_t first = table.first_tile[t.r.worker];
            const double norm = norm_of<kThreads>(a, first, table.first_tile[t.r.worker + 1], sums);
            if (tile == first && threadIdx.x == 0 && a.norm) a.norm[t.r.worker] = (float)norm;
            return factor_of(norm, a.max_norm);
        }
    };
    of_dtype(t.r.dtype, [&](auto kind) {
        using T = decltype(kind);
        T* data = static_cast<T*>(t.r.data) + t.from;
        if (a.out) scale<ONCE>(data, a.out + t.r.worker * a.out_ld + t.r.column + t.from, t.n, factor);
        else scale<ONCE>(data, data, t.n, factor);
    });
}

template <typename F>
void over_tiles(ClipShape& a, F launch) {
    for (a.tile0 = 0; a.tile0 < a.g.tiles; a.tile0 += kTilesOfLaunch)
        launch(dim3((unsigned)(a.g.tiles - a.tile0 < kTilesOfLaunch ? a.g.tiles - a.tile0 : kTilesOfLaunch)));
}

// What is read once, or beyond the caches before it is read again, goes past them (non-temporal): norms of 8 x 25.6 million, bf16, 72 -> 65 us, clipping of 32 x 25.6 million, fp32,
// 1807 -> 1738; but of 8 x 1 million, which the caches hold between its two reads, 23 -> 31.
constexpr uint64_t kCachedTiles = 1024;                           // 64 MB of fp32

void launch_squares(ClipShape& a, bool once, hipStream_t stream) {
    over_tiles(a, [&](dim3 grid) {
        if (once) hipLaunchKernelGGL(squares_kernel<true>, grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL(squares_kernel<false>, grid, dim3(kThreads), 0, stream, a);
    });
}
void launch_join(const ClipShape& a, hipStream_t stream) {
    hipLaunchKernelGGL(norm_kernel, dim3((unsigned)a.g.workers), dim3(kJoinThreads), 0, stream, a);
}

ClipShape shape_of(const ClipArgs& args) {
    ClipShape a{};
    static_cast<ClipArgs&>(a) = args;
    a.squares = static_cast<double*>(a.work);
    return a;
}

}  // namespace

hipError_t launch_lay(const ds_gradients& g, const RecordBatch& batch, hipStream_t stream) {
    hipLaunchKernelGGL(lay_kernel, dim3((unsigned)batch.here), dim3(kThreads), 0, stream, g, batch);
    return hipGetLastError();
}

uint64_t gradient_norm_work_bytes(const ds_gradients& g) { return g.tiles * sizeof(double); }

hipError_t launch_gradient_norm(const ClipArgs& args, hipStream_t stream) {
    ClipShape a = shape_of(args);
    launch_squares(a, true, stream);
    launch_join(a, stream);
    return hipGetLastError();
}

uint64_t clip_work_bytes(const ds_gradients& g) { return (g.tiles + g.workers) * sizeof(double); }

hipError_t launch_clip(const ClipArgs& args, hipStream_t stream) {
    ClipShape a = shape_of(args);
    const bool once = a.g.tiles > kCachedTiles;
    launch_squares(a, once, stream);
    // Few tiles a worker: a launch saved (4 x 30011, fp32, 15.9 -> 13.6 us).  A worker without tiles has no workgroup to write its norm.
    const bool joined = a.g.worker_tiles > 2 * kThreads || a.g.worker_tiles * a.g.workers != a.g.tiles || a.g.tiles == 0;
    if (joined) {
        a.factor = a.squares + a.g.tiles;
        launch_join(a, stream);
    }
    over_tiles(a, [&](dim3 grid) {
        if (once && joined) hipLaunchKernelGGL((scale_kernel<true, true>), grid, dim3(kThreads), 0, stream, a);
        else if (once) hipLaunchKernelGGL((scale_kernel<true, false>), grid, dim3(kThreads), 0, stream, a);
        else if (joined) hipLaunchKernelGGL((scale_kernel<false, true>), grid, dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL((scale_kernel<false, false>), grid, dim3(kThreads), 0, stream, a);
    });
    return hipGetLastError();
}

}  // namespace dsq
