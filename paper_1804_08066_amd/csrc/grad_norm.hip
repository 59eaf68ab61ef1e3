// The L2 norm of a model's gradients, all tensors together, and the gradients scaled to a given norm.
//
//   norm = sqrt(sum over tensors and values of x^2);  c = 1 where norm <= max_norm, else fl(max_norm / norm);  y = x * c
//
// The squares are added in fp64: the squares of all three types' values are exact there (and cannot overflow), and a sum over
// 10^9 of them keeps ten digits, which a model sharded over several GPUs needs to combine its shards' norms.  Every
// workgroup stores one partial sum, whose order of additions is a function of the tensors' sizes alone, and the partial sums
// are added in a fixed order: equal inputs give equal bits.  Both passes are bound by memory: the norm reads every value
// once, clipping reads it once more and writes it.

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "values.h"

namespace mqg {
namespace {

using namespace values;

constexpr uint32_t kThreads = 256;
// Values of a tensor that a workgroup takes at a time.  (1.2 G half-precision values clipped into fp32, pieces of 2048, 4096, 8192 and
// 16384: 1645, 1567, 1677 and 1648 us.)
constexpr uint32_t kPiece = 4096;

// which of the tensors a piece belongs to: starts[k] <= piece < starts[k + 1], as in tensor_of_block, for more than 64
template <uint32_t ENTRIES>
__device__ __forceinline__ uint32_t tensor_of_piece(const uint32_t (&starts)[ENTRIES], const uint32_t count, const uint32_t piece) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t passed = 0;
#pragma unroll
    for (uint32_t first = 0; first < ENTRIES; first += 64u) {
        const uint32_t i = first + lane;
        const uint32_t start = starts[i < ENTRIES ? i : ENTRIES - 1u];
        passed += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(i < count && start <= piece));
    }
    return passed - 1u;   // starts[0] is 0: at least one
}

// this lane's share of the squares of x[0 .. count), count <= kPiece; ONCE: with streaming loads
template <int DTYPE, bool ONCE>
__device__ __forceinline__ double piece_squares(const void* x, const uint32_t count) {
    constexpr int V = DTYPE == kF32 ? 4 : 8;
    constexpr uint32_t kRow = kThreads * V, kRows = kPiece / kRow;
    double acc = 0.0;
    if (count == kPiece) {
        Pack<DTYPE, V> t[kRows];
#pragma unroll
        for (uint32_t r = 0; r < kRows; ++r) {
            if constexpr (ONCE) t[r].load_once(at<DTYPE>(x, r * kRow + threadIdx.x * V));
            else t[r].load(at<DTYPE>(x, r * kRow + threadIdx.x * V));
        }
#pragma unroll
        for (uint32_t r = 0; r < kRows; ++r) {
            float v[V];
            t[r].get(v);
#pragma unroll
            for (int i = 0; i < V; ++i) acc = __builtin_fma((double)v[i], (double)v[i], acc);
        }
        return acc;
    }
    for (uint32_t i = threadIdx.x; i < count; i += kThreads) {
        const double v = (double)load_one<DTYPE>(x, i);
        acc = __builtin_fma(v, v, acc);
    }
    return acc;
}

// the sum over the workgroup, in every lane
__device__ __forceinline__ double workgroup_sum(double acc) {
    __shared__ double s_part[kThreads / 64u];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) acc += __shfl_xor(acc, m, 64);
    if ((threadIdx.x & 63u) == 0u) s_part[threadIdx.x >> 6] = acc;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 64u; ++w) t += s_part[w];
    return t;
}

// The workgroups take pieces in turn: a partial sum of each.
template <bool ONCE, class Table>
__global__ __launch_bounds__(kThreads) void norm_partial_kernel(const Table b, double* __restrict__ partials) {
    double acc = 0.0;
    for (uint32_t piece = blockIdx.x; piece < b.pieces; piece += gridDim.x) {
        const uint32_t k = tensor_of_piece(b.start, b.count, piece);
        const uint64_t base = (uint64_t)(piece - b.start[k]) * kPiece;
        const uint64_t left = b.n[k] - base;
        const uint32_t count = left < kPiece ? (uint32_t)left : kPiece;
        const void* x = b.data[k];
        acc += with_dtype(b.dtype[k], [&](auto d) { return piece_squares<d, ONCE>(at<d>(x, base), count); });
    }
    const double t = workgroup_sum(acc);
    if (threadIdx.x == 0u) partials[blockIdx.x] = t;
}

// in every lane of the workgroup
__device__ __forceinline__ double norm_of_partials(const double* __restrict__ partials, const uint32_t count) {
    double acc = 0.0;
    constexpr uint32_t kAhead = 8;
    for (uint32_t i = threadIdx.x; i < count; i += kAhead * kThreads) {
        double t[kAhead];
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) t[j] = i + j * kThreads < count ? partials[i + j * kThreads] : 0.0;
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) acc += t[j];
    }
    return __builtin_sqrt(workgroup_sum(acc));
}
__global__ __launch_bounds__(kThreads) void norm_finish_kernel(const double* __restrict__ partials, const uint32_t count, double* __restrict__ norm) {
    const double n = norm_of_partials(partials, count);
    if (threadIdx.x == 0u) *norm = n;
}

// a norm that is not a number makes the factor one too: nothing hides it
__device__ __forceinline__ float clip_factor(double norm, double max_norm) { return norm <= max_norm ? 1.0f : (float)(max_norm / norm); }

// factor() is asked for when the values are on their way.  In place, a factor of 1 leaves every value as it is: nothing is written.
template <int IN, int OUT, class F>
__device__ __forceinline__ void clip_piece(const void* x, void* y, const uint32_t count, F factor) {
    constexpr int V = IN == kF32 || OUT == kF32 ? 4 : 8;
    constexpr uint32_t kRow = kThreads * V, kRows = kPiece / kRow;
    if (count == kPiece) {
        Pack<IN, V> t[kRows];
#pragma unroll
        for (uint32_t r = 0; r < kRows; ++r) t[r].load_once(at<IN>(x, r * kRow + threadIdx.x * V));
        const float c = factor();
        if (c == 1.0f && x == y) return;
#pragma unroll
        for (uint32_t r = 0; r < kRows; ++r) {
            float v[V];
            t[r].get(v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] *= c;
            Pack<OUT, V> o;
            o.set(v);
            o.store_once(at<OUT>(y, r * kRow + threadIdx.x * V));
        }
        return;
    }
    const float c = factor();
    if (c == 1.0f && x == y) return;
    for (uint32_t i = threadIdx.x; i < count; i += kThreads) store_one<OUT>(y, i, load_one<IN>(x, i) * c);
}

// A workgroup for every piece.  (2048 that take pieces in turn: 1745 us instead of 1677 for 1.2 G values in pieces of 8192.)
// FEW: `few` partial sums stand in for the norm, and every workgroup adds them up as norm_finish_kernel does; the first leaves the norm
// in *norm.  Otherwise a norm that clips nothing ends the work in place before a value is read.
template <bool FEW, class Table>
__global__ __launch_bounds__(kThreads) void clip_kernel(const Table b, const double* __restrict__ partials, const uint32_t few, double* __restrict__ norm,
                                                        const double max_norm) {
    float c = FEW ? 0.0f : clip_factor(*norm, max_norm);
    bool have = !FEW;
    const auto factor = [&] {
        if (FEW && !have) {
            const double n = norm_of_partials(partials, few);
            if (blockIdx.x == 0u && threadIdx.x == 0u) *norm = n;
            c = clip_factor(n, max_norm);
            have = true;
        }
        return c;
    };
    for (uint32_t piece = blockIdx.x; piece < b.pieces; piece += gridDim.x) {
        const uint32_t k = tensor_of_piece(b.start, b.count, piece);
        const uint64_t base = (uint64_t)(piece - b.start[k]) * kPiece;
        const uint64_t left = b.n[k] - base;
        const uint32_t count = left < kPiece ? (uint32_t)left : kPiece;
        const void* x = b.data[k];
        void* y = b.out[k];
        if (!FEW && c == 1.0f && x == y) continue;   // every value is its own
        with_dtype(b.dtype[k], [&](auto in) {
            with_dtype(b.out_dtype[k], [&](auto out) { clip_piece<in, out>(at<in>(x, base), at<out>(y, base), count, factor); });
        });
    }
}

constexpr uint32_t kMaxBlocks = 1u << 23;   // a launch holds less than 2^32 lanes
// So few partial sums are added up by every one of so few workgroups of the clipping kernel, without a launch in between (half-precision
// values into fp32: 3 M in ten tensors 13.2 -> 8.9 us, 8 M in sixty 20.9 -> 16.6, 40 M 56 -> 51; into half precision 13.7 -> 8.3, 18.1 -> 15.5,
// 41.5 -> 42.3; 234 M into fp32 286 -> 299).
// In place a piece counts as kInPlace: with the norm at hand first, one that clips nothing ends the work there before a value is read
// (half precision, without and with that launch: 15 M 14.2 and 16.0 us, 20 M 18.1 and 15.1, 60 M 44.6 and 27.8; 60 M clipped 58.2 and 58.0).
constexpr uint32_t kFewPartials = kNormBlocks, kFewPieces = 16384, kInPlace = 4;

// fills `b` with the tensors from items[first] on, as many as fit; returns the next one
template <class Table, class F>
uint32_t fill_table(Table& b, const mqg_clip_item* items, uint32_t first, uint32_t count, F entry) {
    uint64_t pieces = 0;
    uint32_t i = first;
    b.count = 0;
    for (; i < count && b.count < Table::kTensors; ++i) {
        if (items[i].n == 0) continue;
        b.start[b.count] = (uint32_t)pieces;
        b.data[b.count] = items[i].data;
        b.n[b.count] = items[i].n;
        b.dtype[b.count] = (uint8_t)items[i].dtype;
        entry(b.count, items[i]);
        ++b.count;
        pieces += (items[i].n + kPiece - 1u) / kPiece;
    }
    b.pieces = (uint32_t)pieces;
    return i;
}

}  // namespace

uint64_t norm_max_values() { return ((uint64_t)0x7FFFFFFF - MQG_MAX_NORM_TENSORS) * kPiece; }   // pieces of a launch fit 31 bits

// the partial sums of all tensors; *stored: how many
template <class Table>
static hipError_t launch_partials(const mqg_clip_item* items, uint32_t count, bool once, double* partials, uint32_t* stored, hipStream_t stream) {
    Table b;
    *stored = 0;
    for (uint32_t i = 0; i < count;) {
        i = fill_table(b, items, i, count, [](uint32_t, const mqg_clip_item&) {});
        if (b.pieces == 0) continue;
        const uint32_t blocks = std::min(b.pieces, kNormBlocks);
        hipLaunchKernelGGL((once ? norm_partial_kernel<true, Table> : norm_partial_kernel<false, Table>), dim3(blocks), dim3(kThreads), 0, stream, b, partials + *stored);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        *stored += blocks;
    }
    return hipSuccess;
}
static hipError_t launch_partials(const mqg_clip_item* items, uint32_t count, bool once, double* partials, uint32_t* stored, hipStream_t stream) {
    return count <= NormTableFew::kTensors ? launch_partials<NormTableFew>(items, count, once, partials, stored, stream)
                                           : launch_partials<NormTable>(items, count, once, partials, stored, stream);
}
static hipError_t launch_finish(const double* partials, uint32_t stored, double* norm, hipStream_t stream) {
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kThreads), 0, stream, partials, stored, norm);
    return hipGetLastError();
}

hipError_t launch_global_norm(const mqg_clip_item* items, uint32_t count, double* partials, double* norm, hipStream_t stream) {
    uint32_t stored;
    const hipError_t e = launch_partials(items, count, true, partials, &stored, stream);
    return e == hipSuccess ? launch_finish(partials, stored, norm, stream) : e;
}

template <class Table>
static hipError_t launch_clip_pieces(const mqg_clip_item* items, uint32_t count, const double* partials, uint32_t few, double* norm, double max_norm,
                                     hipStream_t stream) {
    Table b;
    for (uint32_t i = 0; i < count;) {
        i = fill_table(b, items, i, count, [&](uint32_t k, const mqg_clip_item& it) {
            b.out[k] = it.out;
            b.out_dtype[k] = (uint8_t)it.out_dtype;
        });
        if (b.pieces == 0) continue;
        hipLaunchKernelGGL((few != 0u ? clip_kernel<true, Table> : clip_kernel<false, Table>), dim3(std::min(b.pieces, kMaxBlocks)), dim3(kThreads), 0, stream, b, partials, few, norm, max_norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        few = 0;   // the first launch has left the norm
    }
    return hipSuccess;
}

static hipError_t launch_clip_pieces(const mqg_clip_item* items, uint32_t count, const double* partials, uint32_t few, double* norm, double max_norm,
                                     hipStream_t stream) {
    return count <= ClipTableFew::kTensors ? launch_clip_pieces<ClipTableFew>(items, count, partials, few, norm, max_norm, stream)
                                           : launch_clip_pieces<ClipTable>(items, count, partials, few, norm, max_norm, stream);
}

hipError_t launch_clip(const mqg_clip_item* items, uint32_t count, const double* norm, double max_norm, hipStream_t stream) {
    return launch_clip_pieces(items, count, nullptr, 0, const_cast<double*>(norm), max_norm, stream);   // which is only read
}

hipError_t launch_clip_global_norm(const mqg_clip_item* items, uint32_t count, double max_norm, double* partials, double* norm, hipStream_t stream) {
    uint64_t bytes = 0, pieces = 0;
    for (uint32_t i = 0; i < count; ++i) {
        bytes += items[i].n * bytes_of(items[i].dtype);
        pieces += (items[i].n + kPiece - 1u) / kPiece * (items[i].data == items[i].out ? kInPlace : 1u);
    }
    // Values that clipping may find in the last-level cache are read with ordinary loads: 0.2, 0.5 and 0.8 GB of half-precision values into
    // fp32 took 182, 308 and 686 us with streaming loads and take 170, 291 and 676; 2.4 GB 1567 and 1580.
    uint32_t stored;
    hipError_t e = launch_partials(items, count, bytes > (1ull << 30), partials, &stored, stream);
    if (e != hipSuccess) return e;
    const bool few = stored > 0 && stored <= kFewPartials && pieces <= kFewPieces;
    if (!few) e = launch_finish(partials, stored, norm, stream);
    return e == hipSuccess ? launch_clip_pieces(items, count, partials, few ? stored : 0u, norm, max_norm, stream) : e;
}

}  // namespace mqg
