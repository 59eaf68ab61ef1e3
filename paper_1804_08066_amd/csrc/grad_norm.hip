// The L2 norm of a model's gradients, all tensors together, and the gradients scaled to a given norm.
//
//   norm = sqrt(sum over tensors and values of x^2);  c = 1 where norm <= max_norm, else fl(max_norm / norm);  y = x * c
//
// The squares are added in fp64: the squares of all three types' values are exact there (and cannot overflow), and a sum over
// 10^9 of them keeps ten digits, which a model sharded over several GPUs needs to combine its shards' norms.  Every
// workgroup stores one partial sum, whose order of additions is a function of the tensors' sizes alone, and the partial sums
// are added in a fixed order: equal inputs give equal bits.  Both passes are bound by memory: the norm reads every value
// once, clipping reads it once more and writes it.

#include <type_traits>

#include "kernels.h"
#include "values.h"

namespace mqg {
namespace {

using namespace values;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kPiece = 8192;   // values of a tensor that a workgroup takes at a time

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

// this lane's share of the squares of x[0 .. count), count <= kPiece
template <int DTYPE>
__device__ __forceinline__ double piece_squares(const void* x, const uint32_t count) {
    constexpr int V = DTYPE == kF32 ? 4 : 8;
    constexpr uint32_t kRow = kThreads * V, kRows = kPiece / kRow;
    double acc = 0.0;
    if (count == kPiece) {
        Pack<DTYPE, V> t[kRows];
#pragma unroll
        for (uint32_t r = 0; r < kRows; ++r) t[r].load_once(at<DTYPE>(x, r * kRow + threadIdx.x * V));
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

__global__ __launch_bounds__(kThreads) void norm_partial_kernel(const NormTable b, double* __restrict__ partials) {
    double acc = 0.0;
    for (uint32_t piece = blockIdx.x; piece < b.pieces; piece += gridDim.x) {
        const uint32_t k = tensor_of_piece(b.start, b.count, piece);
        const uint64_t base = (uint64_t)(piece - b.start[k]) * kPiece;
        const uint64_t left = b.n[k] - base;
        const uint32_t count = left < kPiece ? (uint32_t)left : kPiece;
        const void* x = b.data[k];
        acc += with_dtype(b.dtype[k], [&](auto d) { return piece_squares<d>(at<d>(x, base), count); });
    }
    const double t = workgroup_sum(acc);
    if (threadIdx.x == 0u) partials[blockIdx.x] = t;
}

__global__ __launch_bounds__(kThreads) void norm_finish_kernel(const double* __restrict__ partials, const uint32_t count, double* __restrict__ norm) {
    double acc = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += kThreads) acc += partials[i];
    const double t = workgroup_sum(acc);
    if (threadIdx.x == 0u) *norm = __builtin_sqrt(t);
}

// a norm that is not a number makes the factor one too: nothing hides it
__device__ __forceinline__ float clip_factor(double norm, double max_norm) { return norm <= max_norm ? 1.0f : (float)(max_norm / norm); }

template <int IN, int OUT>
__device__ __forceinline__ void clip_piece(const void* x, void* y, const uint32_t count, const float c) {
    constexpr int V = IN == kF32 || OUT == kF32 ? 4 : 8;
    constexpr uint32_t kRow = kThreads * V, kRows = kPiece / kRow;
    if (count == kPiece) {
        Pack<IN, V> t[kRows];
#pragma unroll
        for (uint32_t r = 0; r < kRows; ++r) t[r].load_once(at<IN>(x, r * kRow + threadIdx.x * V));
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
    for (uint32_t i = threadIdx.x; i < count; i += kThreads) store_one<OUT>(y, i, load_one<IN>(x, i) * c);
}

__global__ __launch_bounds__(kThreads) void clip_kernel(const ClipTable b, const double* __restrict__ norm, const double max_norm) {
    const float c = clip_factor(*norm, max_norm);
    for (uint32_t piece = blockIdx.x; piece < b.pieces; piece += gridDim.x) {
        const uint32_t k = tensor_of_piece(b.start, b.count, piece);
        const uint64_t base = (uint64_t)(piece - b.start[k]) * kPiece;
        const uint64_t left = b.n[k] - base;
        const uint32_t count = left < kPiece ? (uint32_t)left : kPiece;
        const void* x = b.data[k];
        void* y = b.out[k];
        with_dtype(b.dtype[k], [&](auto in) {
            with_dtype(b.out_dtype[k], [&](auto out) { clip_piece<in, out>(at<in>(x, base), at<out>(y, base), count, c); });
        });
    }
}

uint32_t blocks_of(uint32_t pieces) { return pieces < kNormBlocks ? pieces : kNormBlocks; }

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

hipError_t launch_global_norm(const mqg_clip_item* items, uint32_t count, double* partials, double* norm, hipStream_t stream) {
    NormTable b;
    uint32_t stored = 0;
    for (uint32_t i = 0; i < count;) {
        i = fill_table(b, items, i, count, [](uint32_t, const mqg_clip_item&) {});
        if (b.pieces == 0) continue;
        const uint32_t blocks = blocks_of(b.pieces);
        hipLaunchKernelGGL(norm_partial_kernel, dim3(blocks), dim3(kThreads), 0, stream, b, partials + stored);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        stored += blocks;
    }
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kThreads), 0, stream, partials, stored, norm);
    return hipGetLastError();
}

hipError_t launch_clip(const mqg_clip_item* items, uint32_t count, const double* norm, double max_norm, hipStream_t stream) {
    ClipTable b;
    for (uint32_t i = 0; i < count;) {
        i = fill_table(b, items, i, count, [&](uint32_t k, const mqg_clip_item& it) {
            b.out[k] = it.out;
            b.out_dtype[k] = (uint8_t)it.out_dtype;
        });
        if (b.pieces == 0) continue;
        hipLaunchKernelGGL(clip_kernel, dim3(blocks_of(b.pieces)), dim3(kThreads), 0, stream, b, norm, max_norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace mqg
