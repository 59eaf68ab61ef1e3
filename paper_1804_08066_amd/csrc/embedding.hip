// Rows of a table by token, and the gradient of the table.
//
// The gradient is added up by sorted tokens: the positions are sorted by their row (a stable radix sort, so that positions of
// one row keep their order), and the rows of grad_out that belong to one row of the table are then a run of that order.  No
// atomic adds a floating value, so equal inputs give equal bits.

#include <algorithm>
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
    const uint32_t col = ((blockIdx.y << shift) + lane) * V;
    if (col >= dim) return;
    for (uint64_t p = (uint64_t)blockIdx.x * (kThreads >> shift) + (threadIdx.x >> shift); p < ids.count; p += (uint64_t)gridDim.x * (kThreads >> shift)) {
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
        } else {
            for (uint32_t i = 0; col + i < dim; ++i) store_one<OUT>(y, i, there ? load_one<IN>(x, i) * scale : 0.0f);
        }
    }
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
    uint4* named;             // first pass of a gradient that is overwritten: [rows] bytes, cleared by the count and set by the scatter
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
    if (a.named != nullptr) {
        const uint64_t all = (a.rows + 15u) / 16u;
        for (uint64_t i = (uint64_t)blockIdx.x * kSortThreads + threadIdx.x; i < all; i += (uint64_t)gridDim.x * kSortThreads) a.named[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (blockIdx.x >= a.ranges) return;
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
            if (a.named != nullptr && key[j] < a.rows) reinterpret_cast<uint8_t*>(a.named)[key[j]] = 1u;
        }
    }
}

template <int OUT, int V>
__device__ __forceinline__ void clear_row(const RowMatrix& out, uint32_t dim, uint64_t row, uint32_t col) {
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
// a table without tokens: all of it is cleared
template <int OUT>
__global__ __launch_bounds__(kThreads) void clear_rows_kernel(const RowMatrix out, const uint32_t dim, const uint32_t shift) {
    constexpr int V = OUT == kF32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & ((1u << shift) - 1u);
    const uint32_t col = ((blockIdx.y << shift) + lane) * V;
    if (col >= dim) return;
    for (uint64_t row = (uint64_t)blockIdx.x * (kThreads >> shift) + (threadIdx.x >> shift); row < out.rows; row += (uint64_t)gridDim.x * (kThreads >> shift)) {
        clear_row<OUT, V>(out, dim, row, col);
    }
}

// ---- the sums ------------------------------------------------------------------------------------------
// The sorted positions are cut into chunks, and the lanes of a chunk add up its runs, eight rows of grad_out in flight.  A run
// that starts in a chunk and ends in the next one is added up by the chunk it starts in; one that goes on into the chunk after
// that is long: each of its chunks leaves a partial sum, which join_runs_kernel adds up in the order of the chunks.  So a row
// of the table that half a batch names is read by as many workgroups as any other half, and every chunk can tell from the
// keys around it which of its runs are whose.
constexpr uint32_t kRows = 8;            // in flight

struct SumArgs {
    const uint32_t *keys, *order;
    uint64_t count;                       // positions
    RowMatrix grad, out;
    float* partials;                      // [chunks][2][width]: of the long run that a chunk begins in, and of the one that begins in it
    const uint8_t* named;                 // [rows], rows that a position names; nullptr: rows that none names are left as they are
    uint32_t dim, width, shift, chunk;    // width: dim, rounded up to 8; 1 << shift lanes hold a row or a slice of it
    uint32_t chunk_blocks;                // workgroups of chunks; the others clear rows
    float scale;
    bool accumulate;
};

// the next chunk's positions [start, ...) continue a run of key `k` that starts before them: is that run long?
__device__ __forceinline__ bool continues_long(const SumArgs& a, uint64_t start, uint32_t k) {
    const bool began_before = start > a.chunk && a.keys[start - a.chunk - 1u] == k;
    return began_before || (start + a.chunk < a.count && a.keys[start + a.chunk] == k);
}

template <int OUT, int V>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, uint32_t col, const float (&sum)[V]) {
    void* y = at<OUT>(a.out.data, (uint64_t)row * a.out.stride + col);
    if (col + V <= a.dim) {
        float v[V];
        Pack<OUT, V> o;
        if (a.accumulate) {
            o.load(y);
            o.get(v);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = a.accumulate ? __builtin_fmaf(a.scale, sum[i], v[i]) : a.scale * sum[i];
        o.set(v);
        o.store(y);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (col + i < a.dim) store_one<OUT>(y, i, a.accumulate ? __builtin_fmaf(a.scale, sum[i], load_one<OUT>(y, i)) : a.scale * sum[i]);
    }
}
template <int V>
__device__ __forceinline__ void write_partial(const SumArgs& a, uint64_t chunk, uint32_t slot, uint32_t col, const float (&sum)[V]) {
    float* p = a.partials + (2u * chunk + slot) * a.width + col;   // a whole number of V: width is
    Pack<kF32, V> o;
    o.set(sum);
    o.store(p);
}

// UNIFORM: a wave's lanes all belong to one chunk, whose keys are then scalar loads
template <int IN, int OUT, bool UNIFORM>
__global__ __launch_bounds__(kThreads) void sum_runs_kernel(const SumArgs a) {
    constexpr int V = IN == kF32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & ((1u << a.shift) - 1u);
    const uint32_t col = ((blockIdx.y << a.shift) + lane) * V;
    if (col >= a.dim) return;
    if (blockIdx.x >= a.chunk_blocks) {
        uint64_t row = (uint64_t)(blockIdx.x - a.chunk_blocks) * (kThreads >> a.shift) + (threadIdx.x >> a.shift);
        for (; row < a.out.rows; row += (uint64_t)(gridDim.x - a.chunk_blocks) * (kThreads >> a.shift)) {
            if (a.named[row] == 0u) clear_row<OUT, V>(a.out, a.dim, row, col);
        }
        return;
    }
    uint32_t c = blockIdx.x * (kThreads >> a.shift) + (threadIdx.x >> a.shift);
    if constexpr (UNIFORM) c = (uint32_t)__builtin_amdgcn_readfirstlane((int)c);
    const uint64_t start = (uint64_t)c * a.chunk, end = min(start + a.chunk, a.count);
    if (start >= a.count) return;
    uint32_t cur = a.keys[start];
    const uint32_t rows = (uint32_t)a.out.rows;
    if (cur >= rows) return;                               // keys rise: no position from here on adds to a row
    const uint32_t last = a.keys[end - 1u];                // a run of this key may go on behind the chunk
    bool skip = false, head = false;                       // of the run that began before this chunk
    if (start > 0u && a.keys[start - 1u] == cur) {
        head = continues_long(a, start, cur);
        skip = !head;
    }
    const bool tail = end < a.count && continues_long(a, end, last);   // where the last key's run goes on at all
    const uint32_t beyond = tail ? rows : last;            // key whose positions behind the chunk belong to it: `rows` for none
    float sum[V] = {};
    const auto finish = [&](bool ends) {                   // the run of `cur`, which ends here or goes on behind the chunk
        if (head) write_partial<V>(a, c, 0u, col, sum);
        else if (!ends && tail) write_partial<V>(a, c, 1u, col, sum);
        else if (!skip) write_row<OUT, V>(a, cur, col, sum);
    };
    const bool whole = col + V <= a.dim;
    for (uint64_t i = start;; i += kRows) {
        uint32_t key[kRows];
        bool valid[kRows];
        Pack<IN, V> t[kRows];
#pragma unroll
        for (uint32_t j = 0; j < kRows; ++j) {
            const bool in = i + j < a.count;
            key[j] = in ? a.keys[i + j] : rows;
            valid[j] = in && key[j] < rows && (i + j < end || key[j] == beyond);
        }
#pragma unroll
        for (uint32_t j = 0; j < kRows; ++j) {
            if (!valid[j] || (skip && key[j] == cur)) continue;
            const void* x = at<IN>(a.grad.data, (uint64_t)a.order[i + j] * a.grad.stride + col);
            if (whole) {
                t[j].load(x);
            } else {
                float v[V];
#pragma unroll
                for (int l = 0; l < V; ++l) v[l] = col + l < a.dim ? load_one<IN>(x, l) : 0.0f;
                t[j].set(v);
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < kRows; ++j) {
            if (!valid[j]) {
                finish(i + j < end || key[j] != last);
                return;
            }
            if (key[j] != cur) {
                finish(true);
                cur = key[j];
                head = skip = false;
#pragma unroll
                for (int l = 0; l < V; ++l) sum[l] = 0.0f;
            }
            if (!skip) {
                float v[V];
                t[j].get(v);
#pragma unroll
                for (int l = 0; l < V; ++l) sum[l] += v[l];
            }
        }
    }
}

// The partial sums of the long run that begins in a chunk: the waves take them in turn, and add up theirs in order.
constexpr uint32_t kJoinWaves = 8, kJoinThreads = 64u * kJoinWaves;
template <int OUT>
__global__ __launch_bounds__(kJoinThreads) void join_runs_kernel(const SumArgs a) {
    __shared__ float s_sum[kJoinWaves][64][4];
    const uint64_t c = blockIdx.x, start = c * a.chunk, end = start + a.chunk;
    if (end >= a.count) return;
    const uint32_t k = a.keys[end];
    if (k >= a.out.rows || a.keys[end - 1u] != k || (start > 0u && a.keys[start - 1u] == k) || !continues_long(a, end, k)) return;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = (blockIdx.y * 64u + lane) * 4u;
    // chunks behind this one that begin in the run: a search by 64 at a time
    const uint64_t most = (a.count - 1u) / a.chunk - c;
    uint64_t low = 2, high = most + 1u;                    // chunk c + low - 1 begins in it, chunk c + high does not
    while (low < high) {
        const uint64_t step = (high - low + 63u) / 64u, probe = low + lane * step;
        const bool in = probe < high && a.keys[(c + probe) * a.chunk] == k;
        const uint32_t seen = (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
        if (seen == 0u) break;
        const uint64_t found = low + (uint64_t)(seen - 1u) * step;   // begins in it
        high = min(high, found + step);
        low = found + 1u;
    }
    const uint64_t parts = low;                            // slot 1 of c, slot 0 of c + 1 .. c + low - 1
    float sum[4] = {};
    if (col < a.width) {
        constexpr uint32_t kAhead = 4;
        for (uint64_t p = wave; p < parts; p += kAhead * kJoinWaves) {
            Pack<kF32, 4> t[kAhead];
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) {
                const uint64_t q = p + j * kJoinWaves;
                if (q < parts) t[j].load(a.partials + (2u * (c + q) + (q == 0u ? 1u : 0u)) * a.width + col);
            }
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) {
                if (p + j * kJoinWaves >= parts) continue;
                float v[4];
                t[j].get(v);
#pragma unroll
                for (int l = 0; l < 4; ++l) sum[l] += v[l];
            }
        }
    }
#pragma unroll
    for (int l = 0; l < 4; ++l) s_sum[wave][lane][l] = sum[l];
    __syncthreads();
    if (wave != 0u || col >= a.dim) return;
#pragma unroll
    for (uint32_t w = 1; w < kJoinWaves; ++w) {
#pragma unroll
        for (int l = 0; l < 4; ++l) sum[l] += s_sum[w][lane][l];
    }
    write_row<OUT, 4>(a, k, col, sum);
}

// lanes that hold a row, as a power of two of at most a workgroup, and slices of a row
uint32_t row_shift(uint32_t dim, uint32_t v) {
    uint32_t shift = 0;
    while ((1u << shift) < kThreads && (1u << shift) * v < dim) ++shift;
    return shift;
}
constexpr uint64_t kMaxBlocks = 1u << 22;   // a launch holds less than 2^32 lanes: the workgroups take rows in turn from there on
dim3 row_grid(uint64_t rows, uint32_t dim, uint32_t v) {
    const uint32_t shift = row_shift(dim, v), per = kThreads >> shift, width = v << shift;
    return dim3((uint32_t)std::min<uint64_t>((rows + per - 1u) / per, kMaxBlocks), (dim + width - 1u) / width);
}

// Positions of a chunk: enough chunks to fill the GPU, as long as that allows (a long run leaves a partial sum in every chunk).
uint32_t chunk_of(uint64_t tokens, uint32_t dim) {
    const uint64_t waves = tokens * ((dim + 511u) / 512u);
    uint32_t chunk = 8;
    while (chunk < 64u && waves / (2u * chunk) >= 4096u) chunk *= 2u;
    while (tokens / chunk >= kMaxBlocks) chunk *= 2u;
    return chunk;
}

struct GradWorkspace {
    uint32_t *keys[2], *order[2], *counts, *named;
    float* partials;
    size_t bytes;
};
GradWorkspace grad_workspace(void* base, uint64_t tokens, uint32_t dim, uint64_t rows) {
    GradWorkspace w = {};
    w.named = static_cast<uint32_t*>(base);
    w.bytes = (rows + 15u) & ~(uint64_t)15u;
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
    const uint32_t chunk = chunk_of(tokens, dim);
    w.partials = reinterpret_cast<float*>(take((tokens + chunk - 1u) / chunk * 2u * ((dim + 7u) & ~7u)));
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

size_t embedding_grad_workspace(uint64_t tokens, uint32_t dim, uint64_t rows) { return tokens == 0 ? 0 : grad_workspace(nullptr, tokens, dim, rows).bytes; }

hipError_t launch_embedding_grad(const RowMatrix& grad_out, const TokenIds& ids, uint32_t dim, float scale, const RowMatrix& table_grad,
                                 bool accumulate, void* workspace, hipStream_t stream) {
    SumArgs b = {};
    b.count = ids.count;
    b.grad = grad_out;
    b.out = table_grad;
    b.dim = dim;
    b.width = (dim + 7u) & ~7u;
    b.scale = scale;
    b.accumulate = accumulate;
    hipError_t e = hipSuccess;
    if (ids.count == 0) {
        if (accumulate) return e;
        with_dtype(table_grad.dtype, [&](auto o) {
            constexpr uint32_t v = o == kF32 ? 4u : 8u;
            hipLaunchKernelGGL((clear_rows_kernel<o>), row_grid(table_grad.rows, dim, v), dim3(kThreads), 0, stream, table_grad, dim, row_shift(dim, v));
        });
        return hipGetLastError();
    }
    const GradWorkspace w = grad_workspace(workspace, ids.count, dim, table_grad.rows);
    const SortShape s = sort_shape(ids.count, table_grad.rows);
    SortArgs a = {};
    a.ids = ids;
    a.rows = table_grad.rows;
    a.counts = w.counts;
    a.range = s.range;
    a.ranges = s.ranges;
    a.bits = s.bits;
    a.named = accumulate ? nullptr : reinterpret_cast<uint4*>(w.named);
    for (uint32_t pass = 0; pass < s.passes; ++pass) {
        a.keys_out = w.keys[pass & 1u];
        a.order_out = w.order[pass & 1u];
        a.shift = pass * s.bits;
        const uint64_t clearing = a.named == nullptr ? 0 : a.rows / (64u * kSortThreads);   // four 16-byte stores a lane
        const uint32_t count_blocks = (uint32_t)std::max<uint64_t>(s.ranges, std::min<uint64_t>(clearing, 2048));
        hipLaunchKernelGGL((ids.wide ? sort_count_kernel<true> : sort_count_kernel<false>), dim3(count_blocks), dim3(kSortThreads), 0, stream, a);
        hipLaunchKernelGGL((ids.wide ? sort_scatter_kernel<true> : sort_scatter_kernel<false>), dim3(s.ranges), dim3(kSortThreads), 0, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.keys = a.keys_out;
        a.order = a.order_out;
        a.named = nullptr;
    }
    b.keys = a.keys;
    b.order = a.order;
    b.partials = w.partials;
    b.named = accumulate ? nullptr : reinterpret_cast<const uint8_t*>(w.named);
    b.chunk = chunk_of(ids.count, dim);
    const uint64_t chunks = (ids.count + b.chunk - 1u) / b.chunk;
    with_dtype(grad_out.dtype, [&](auto in) {
        with_dtype(table_grad.dtype, [&](auto o) {
            constexpr uint32_t v = in == kF32 ? 4u : 8u;
            b.shift = row_shift(dim, v);
            dim3 grid = row_grid(chunks, dim, v);
            b.chunk_blocks = grid.x;
            if (!accumulate) grid.x += row_grid(b.out.rows, dim, v).x;
            hipLaunchKernelGGL((b.shift >= 6u ? sum_runs_kernel<in, o, true> : sum_runs_kernel<in, o, false>), grid, dim3(kThreads), 0, stream, b);
        });
    });
    e = hipGetLastError();
    if (e != hipSuccess || chunks < 3u) return e;   // a long run touches three chunks
    with_dtype(table_grad.dtype, [&](auto o) {
        hipLaunchKernelGGL((join_runs_kernel<o>), dim3((uint32_t)chunks, (b.width + 255u) / 256u), dim3(kJoinThreads), 0, stream, b);
    });
    return hipGetLastError();
}

}  // namespace mqg
