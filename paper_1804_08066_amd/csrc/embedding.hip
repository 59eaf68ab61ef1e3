// Rows of a table by token, and the gradient of the table.
//
// The gradient is added up by sorted tokens: the positions are sorted by their row (a stable radix sort, so that positions of
// one row keep their order), and the rows of grad_out that belong to one row of the table are then a run of that order.  No
// atomic adds a floating value, so equal inputs give equal bits.

#include <type_traits>

#include "kernels.h"
#include "values.h"

namespace mqg {
namespace {

using namespace values;

constexpr uint32_t kThreads = 256;

// the row of token i of the table, or `rows` for a token that adds to none
template <bool WIDE>
__device__ __forceinline__ uint32_t row_of(const TokenIds& t, uint64_t i, uint64_t rows, bool padding) {
    const int64_t id = WIDE ? static_cast<const int64_t*>(t.ids)[i] : (int64_t)static_cast<const int32_t*>(t.ids)[i];
    const uint64_t row = (uint64_t)id - (uint64_t)t.first_row;   // one before the first row wraps far beyond the last
    return row < rows && !(padding && id == t.padding) ? (uint32_t)row : (uint32_t)rows;
}

// ---- lookup ------------------------------------------------------------------------------------------
// `1 << shift` lanes hold a row's (or a slice of a row's) values, V each; blockIdx.y: the slice.
template <int IN, int OUT, bool WIDE>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const RowMatrix table, const TokenIds ids, const uint32_t dim, const uint32_t shift,
                                                             const float scale, const RowMatrix out) {
    constexpr int V = IN == kF32 || OUT == kF32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & ((1u << shift) - 1u);
    const uint64_t p = (uint64_t)blockIdx.x * (kThreads >> shift) + (threadIdx.x >> shift);
    const uint32_t col = ((blockIdx.y << shift) + lane) * V;
    if (p >= ids.count || col >= dim) return;
    const uint32_t row = row_of<WIDE>(ids, p, table.rows, false);
    const bool there = row < table.rows;
    const void* x = at<IN>(table.data, (uint64_t)row * table.stride + col);
    void* y = at<OUT>(out.data, p * out.stride + col);
    if (col + V <= dim) {
        float v[V] = {};
        if (there) {
            Pack<IN, V> t;
            t.load(x);
            t.get(v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] *= scale;
        }
        Pack<OUT, V> o;
        o.set(v);
        o.store(y);
        return;
    }
    for (uint32_t i = 0; col + i < dim; ++i) store_one<OUT>(y, i, there ? load_one<IN>(x, i) * scale : 0.0f);
}

// ---- the sort ------------------------------------------------------------------------------------------
// Least significant digit first.  Every workgroup owns a range of the positions; a pass counts each range's digits, and the
// scatter adds up the counts before its own (of smaller digits, and of equal ones in earlier ranges) by itself.
constexpr uint32_t kSortThreads = 256, kSortWaves = kSortThreads / 64u, kSortItems = 8, kSortTile = kSortThreads * kSortItems;
constexpr uint32_t kMaxRanges = 256;     // every workgroup reads all ranges' counts: a few, of any length
constexpr uint32_t kMaxDigitBits = 10;

struct SortShape {
    uint32_t passes, bits, ranges;
    uint64_t range;                       // positions of one, a multiple of kSortTile
};
SortShape sort_shape(uint64_t tokens, uint64_t rows) {
    SortShape s;
    uint32_t all = 1;
    while ((rows >> all) != 0u) ++all;    // keys are 0 .. rows
    s.passes = (all + kMaxDigitBits - 1u) / kMaxDigitBits;
    s.bits = (all + s.passes - 1u) / s.passes;
    const uint64_t tiles = (tokens + kSortTile - 1u) / kSortTile, each = (tiles + kMaxRanges - 1u) / kMaxRanges;
    s.range = each * kSortTile;
    s.ranges = (uint32_t)((tokens + s.range - 1u) / s.range);
    return s;
}

struct SortArgs {
    TokenIds ids;
    uint64_t rows;
    const uint32_t* keys;     // nullptr: the first pass, which reads the tokens
    const uint32_t* order;
    uint32_t* keys_out;
    uint32_t* order_out;
    uint32_t* counts;         // [ranges][1 << bits]
    uint64_t range;
    uint32_t ranges, bits, shift;
};

template <bool WIDE>
__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, uint64_t i) {
    return a.keys != nullptr ? a.keys[i] : row_of<WIDE>(a.ids, i, a.rows, true);
}

template <bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a) {
    __shared__ uint32_t s_count[1u << kMaxDigitBits];
    const uint32_t digits = 1u << a.bits;
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) s_count[d] = 0u;
    __syncthreads();
    const uint64_t first = (uint64_t)blockIdx.x * a.range, end = min(first + a.range, a.ids.count);
    for (uint64_t i = first + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&s_count[(sort_key<WIDE>(a, i) >> a.shift) & (digits - 1u)], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.counts[(uint64_t)blockIdx.x * digits + d] = s_count[d];
}

template <bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const SortArgs a) {
    __shared__ uint32_t s_next[1u << kMaxDigitBits];                    // where the next key of a digit goes
    __shared__ uint32_t s_wave[kSortWaves][1u << kMaxDigitBits];
    __shared__ uint32_t s_total[kSortWaves];
    const uint32_t digits = 1u << a.bits, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;

    // the keys of smaller digits, and of the same digit in earlier ranges; digits of a thread are consecutive
    const uint32_t per = (digits + kSortThreads - 1u) / kSortThreads;   // 1, 2 or 4
    uint32_t before[4] = {}, all[4] = {}, mine = 0;
    for (uint32_t j = 0; j < per; ++j) {
        const uint32_t d = tid * per + j;
        if (d >= digits) break;
        for (uint32_t r = 0; r < a.ranges; ++r) {
            const uint32_t c = a.counts[(uint64_t)r * digits + d];
            if (r < blockIdx.x) before[j] += c;
            all[j] += c;
        }
        mine += all[j];
    }
    uint32_t upto = mine;
#pragma unroll
    for (uint32_t m = 1; m < 64u; m <<= 1) {
        const uint32_t other = __shfl_up(upto, m, 64);
        if (lane >= m) upto += other;
    }
    if (lane == 63u) s_total[wave] = upto;
    __syncthreads();
    uint32_t at = upto - mine;
    for (uint32_t w = 0; w < wave; ++w) at += s_total[w];
    for (uint32_t j = 0; j < per; ++j) {
        const uint32_t d = tid * per + j;
        if (d >= digits) break;
        s_next[d] = at + before[j];
        at += all[j];
    }

    const uint64_t first = (uint64_t)blockIdx.x * a.range, end = min(first + a.range, a.ids.count);
    for (uint64_t tile = first; tile < end; tile += kSortTile) {
        __syncthreads();
        for (uint32_t d = lane; d < digits; d += 64u) s_wave[wave][d] = 0u;
        __builtin_amdgcn_wave_barrier();
        uint32_t key[kSortItems], from[kSortItems], rank[kSortItems];
        bool valid[kSortItems];
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {   // a wave's keys are consecutive, in this order
            const uint64_t i = tile + (uint64_t)wave * (64u * kSortItems) + j * 64u + lane;
            valid[j] = i < end;
            key[j] = valid[j] ? sort_key<WIDE>(a, i) : 0u;
            from[j] = valid[j] && a.order != nullptr ? a.order[i] : (uint32_t)i;
        }
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            const uint32_t d = (key[j] >> a.shift) & (digits - 1u);
            uint64_t same = __builtin_amdgcn_ballot_w64(valid[j]);
            for (uint32_t b = 0; b < a.bits; ++b) {
                const bool one = (d >> b) & 1u;
                const uint64_t ones = __builtin_amdgcn_ballot_w64(one);
                same &= one ? ones : ~ones;
            }
            const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
            uint32_t seen = 0;
            if (valid[j]) {
                seen = __hip_atomic_load(&s_wave[wave][d], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
            }
            __builtin_amdgcn_wave_barrier();
            if (valid[j] && below == 0u) {
                __hip_atomic_store(&s_wave[wave][d], seen + (uint32_t)__builtin_popcountll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
            }
            __builtin_amdgcn_wave_barrier();
            rank[j] = seen + below;
        }
        __syncthreads();
        for (uint32_t d = tid; d < digits; d += kSortThreads) {
            uint32_t next = s_next[d];
#pragma unroll
            for (uint32_t w = 0; w < kSortWaves; ++w) {
                const uint32_t c = s_wave[w][d];
                s_wave[w][d] = next;
                next += c;
            }
            s_next[d] = next;
        }
        __syncthreads();
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            if (!valid[j]) continue;
            const uint32_t to = s_wave[wave][(key[j] >> a.shift) & (digits - 1u)] + rank[j];
            a.keys_out[to] = key[j];
            a.order_out[to] = from[j];
        }
    }
}

// ---- the sums ------------------------------------------------------------------------------------------
template <int OUT>
__global__ __launch_bounds__(kThreads) void clear_rows_kernel(const RowMatrix out, const uint32_t dim, const uint32_t shift) {
    constexpr int V = OUT == kF32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & ((1u << shift) - 1u);
    const uint64_t row = (uint64_t)blockIdx.x * (kThreads >> shift) + (threadIdx.x >> shift);
    const uint32_t col = ((blockIdx.y << shift) + lane) * V;
    if (row >= out.rows || col >= dim) return;
    void* y = at<OUT>(out.data, row * out.stride + col);
    if (col + V <= dim) {
        const float zero[V] = {};
        Pack<OUT, V> o;
        o.set(zero);
        o.store(y);
        return;
    }
    for (uint32_t i = 0; col + i < dim; ++i) store_one<OUT>(y, i, 0.0f);
}

// The lanes of the first position of a run add up the run.
template <int IN, int OUT, bool ACCUMULATE>
__global__ __launch_bounds__(kThreads) void sum_runs_kernel(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ order, const uint64_t count,
                                                            const RowMatrix grad, const uint32_t dim, const uint32_t shift, const float scale, const RowMatrix out) {
    constexpr int V = IN == kF32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & ((1u << shift) - 1u);
    const uint64_t first = (uint64_t)blockIdx.x * (kThreads >> shift) + (threadIdx.x >> shift);
    const uint32_t col = ((blockIdx.y << shift) + lane) * V;
    if (first >= count || col >= dim) return;
    const uint32_t row = keys[first];
    if (row >= out.rows || (first > 0 && keys[first - 1u] == row)) return;
    const uint32_t some = col + V <= dim ? V : dim - col;
    float sum[V] = {};
    for (uint64_t i = first; i < count && keys[i] == row; ++i) {
        const void* x = at<IN>(grad.data, (uint64_t)order[i] * grad.stride + col);
        float v[V] = {};
        if (some == V) {
            Pack<IN, V> t;
            t.load(x);
            t.get(v);
        } else {
            for (uint32_t j = 0; j < some; ++j) v[j] = load_one<IN>(x, j);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += v[j];
    }
    void* y = at<OUT>(out.data, (uint64_t)row * out.stride + col);
    for (uint32_t j = 0; j < some; ++j) store_one<OUT>(y, j, ACCUMULATE ? __builtin_fmaf(scale, sum[j], load_one<OUT>(y, j)) : scale * sum[j]);
}

// lanes that hold a row, as a power of two of at most a workgroup, and slices of a row
uint32_t row_shift(uint32_t dim, uint32_t v) {
    uint32_t shift = 0;
    while ((1u << shift) < kThreads && (1u << shift) * v < dim) ++shift;
    return shift;
}
dim3 row_grid(uint64_t rows, uint32_t dim, uint32_t v) {
    const uint32_t shift = row_shift(dim, v), per = kThreads >> shift, width = v << shift;
    return dim3((uint32_t)((rows + per - 1u) / per), (dim + width - 1u) / width);
}

struct GradWorkspace {
    uint32_t *keys[2], *order[2], *counts;
    size_t bytes;
};
GradWorkspace grad_workspace(void* base, uint64_t tokens, uint64_t rows) {
    GradWorkspace w = {};
    if (tokens == 0) return w;
    const SortShape s = sort_shape(tokens, rows);
    char* p = static_cast<char*>(base);
    const auto take = [&](uint64_t words) {
        uint32_t* at = reinterpret_cast<uint32_t*>(p + w.bytes);
        w.bytes += (words * 4u + 15u) & ~(uint64_t)15u;
        return at;
    };
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = take(tokens);
        w.order[i] = take(tokens);
    }
    w.counts = take((uint64_t)s.ranges << s.bits);
    return w;
}

}  // namespace

hipError_t launch_embedding(const RowMatrix& table, const TokenIds& ids, uint32_t dim, float scale, const RowMatrix& out, hipStream_t stream) {
    if (ids.count == 0) return hipSuccess;
    with_dtype(table.dtype, [&](auto in) {
        with_dtype(out.dtype, [&](auto o) {
            constexpr uint32_t v = in == kF32 || o == kF32 ? 4u : 8u;
            const dim3 grid = row_grid(ids.count, dim, v);
            const uint32_t shift = row_shift(dim, v);
            if (ids.wide) hipLaunchKernelGGL((embedding_kernel<in, o, true>), grid, dim3(kThreads), 0, stream, table, ids, dim, shift, scale, out);
            else hipLaunchKernelGGL((embedding_kernel<in, o, false>), grid, dim3(kThreads), 0, stream, table, ids, dim, shift, scale, out);
        });
    });
    return hipGetLastError();
}

size_t embedding_grad_workspace(uint64_t tokens, uint32_t dim, uint64_t rows) { return grad_workspace(nullptr, tokens, rows).bytes; }

hipError_t launch_embedding_grad(const RowMatrix& grad_out, const TokenIds& ids, uint32_t dim, float scale, const RowMatrix& table_grad,
                                 bool accumulate, void* workspace, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (!accumulate) {
        with_dtype(table_grad.dtype, [&](auto o) {
            constexpr uint32_t v = o == kF32 ? 4u : 8u;
            hipLaunchKernelGGL((clear_rows_kernel<o>), row_grid(table_grad.rows, dim, v), dim3(kThreads), 0, stream, table_grad, dim, row_shift(dim, v));
        });
        e = hipGetLastError();
    }
    if (e != hipSuccess || ids.count == 0) return e;
    const GradWorkspace w = grad_workspace(workspace, ids.count, table_grad.rows);
    const SortShape s = sort_shape(ids.count, table_grad.rows);
    SortArgs a = {};
    a.ids = ids;
    a.rows = table_grad.rows;
    a.counts = w.counts;
    a.range = s.range;
    a.ranges = s.ranges;
    a.bits = s.bits;
    for (uint32_t pass = 0; pass < s.passes; ++pass) {
        a.keys_out = w.keys[pass & 1u];
        a.order_out = w.order[pass & 1u];
        a.shift = pass * s.bits;
        hipLaunchKernelGGL((ids.wide ? sort_count_kernel<true> : sort_count_kernel<false>), dim3(s.ranges), dim3(kSortThreads), 0, stream, a);
        hipLaunchKernelGGL((ids.wide ? sort_scatter_kernel<true> : sort_scatter_kernel<false>), dim3(s.ranges), dim3(kSortThreads), 0, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.keys = a.keys_out;
        a.order = a.order_out;
    }
    with_dtype(grad_out.dtype, [&](auto in) {
        with_dtype(table_grad.dtype, [&](auto o) {
            constexpr uint32_t v = in == kF32 ? 4u : 8u;
            hipLaunchKernelGGL((accumulate ? sum_runs_kernel<in, o, true> : sum_runs_kernel<in, o, false>), row_grid(ids.count, dim, v), dim3(kThreads), 0, stream,
                               a.keys, a.order, ids.count, grad_out, dim, row_shift(dim, v), scale, table_grad);
        });
    });
    return hipGetLastError();
}

}  // namespace mqg
