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

// Values of a row that a lane holds: 16 bytes of the wider type, which are whole lines for a wave.  (Eight values of which
// fp32 are two stores of half a line each: the sums of 131072 half-precision rows took 386 us instead of 345.)
constexpr int values_of(int in, int out) { return in == kF32 || out == kF32 ? 4 : 8; }

// A lane's V values of a row that begin at `col`.  Where fewer are left, the last V of the row: values that two lanes hold are the same
// in both, so that a lane never reads or writes one by one (23694 rows of 455 values: their sums took 28 us with tails that are read
// value by value, and take 12).  Rows of less than V values are read and written one by one.
template <int V>
struct Window {
    uint32_t at, skip;      // first value; those before `col`, which another lane holds too
    bool narrow;
    __device__ __forceinline__ Window(uint32_t col, uint32_t dim) : at(dim < V ? 0u : min(col, dim - V)), skip(col - at), narrow(dim < V) {}
    template <int DTYPE>
    __device__ __forceinline__ void load(Pack<DTYPE, V>& t, const void* row, uint32_t dim) const {
        if (narrow) t.load_some(row, dim);
        else t.load(values::at<DTYPE>(row, at));
    }
    template <int DTYPE>
    __device__ __forceinline__ void load_once(Pack<DTYPE, V>& t, const void* row, uint32_t dim) const {
        if (narrow) t.load_some(row, dim);
        else t.load_once(values::at<DTYPE>(row, at));
    }
    template <int DTYPE>
    __device__ __forceinline__ void store_once(void* row, const float (&v)[V], uint32_t dim) const {
        if (narrow) {
            store_from<DTYPE>(row, v, 0u, dim);
            return;
        }
        Pack<DTYPE, V> o;
        o.set(v);
        o.store_once(values::at<DTYPE>(row, at));
    }
    // the lane's own values only: what is added to an old value is added once
    template <int DTYPE>
    __device__ __forceinline__ void store_own(void* row, const float (&v)[V], uint32_t dim) const {
        if (narrow || skip != 0u) {
            store_from<DTYPE>(values::at<DTYPE>(row, at), v, skip, narrow ? dim : (uint32_t)V);
            return;
        }
        Pack<DTYPE, V> o;
        o.set(v);
        o.store(values::at<DTYPE>(row, at));
    }
    template <int DTYPE>
    static __device__ __forceinline__ void store_from(void* p, const float (&v)[V], uint32_t first, uint32_t end) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if ((uint32_t)i >= first && (uint32_t)i < end) store_one<DTYPE>(p, i, v[i]);
        }
    }
};

// ---- lookup ------------------------------------------------------------------------------------------
// `1 << shift` lanes hold a row's (or a slice of a row's) values, V each, of kLookups rows at a time; the slices of a row are
// neighbouring workgroups.  Bound by the fabric between the caches and memory: 131072 half-precision rows of 4096 values into fp32, 3.2 GB,
// take 530 us.  The rows are written with streaming stores: stores that stay in the caches push the table out of them (40001 rows of 1531
// values, most of them another shard's: 40 us with ordinary stores and a row at a time, 30.5 with streaming ones, 27.7 with two rows).
constexpr uint32_t kLookups = 2;
template <int IN, int OUT, bool WIDE>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const RowMatrix table, const TokenIds ids, const uint32_t dim, const uint32_t shift,
                                                             const uint32_t slices, const float scale, const RowMatrix out) {
    constexpr int V = values_of(IN, OUT);
    const uint32_t lane = threadIdx.x & ((1u << shift) - 1u), per = kThreads >> shift, block = blockIdx.x / slices;
    const uint32_t col = (((blockIdx.x - block * slices) << shift) + lane) * V;
    if (col >= dim) return;
    const Window<V> w(col, dim);
    const uint64_t step = (uint64_t)per * kLookups;
    for (uint64_t p = block * step + (threadIdx.x >> shift); p < ids.count; p += gridDim.x / slices * step) {
        uint32_t row[kLookups];
        bool there[kLookups];
        Pack<IN, V> t[kLookups] = {};
#pragma unroll
        for (uint32_t r = 0; r < kLookups; ++r) {
            row[r] = p + r * per < ids.count ? row_of<WIDE>(ids, p + r * per, table.rows, false) : (uint32_t)table.rows;
            there[r] = row[r] < table.rows;
        }
#pragma unroll
        for (uint32_t r = 0; r < kLookups; ++r) {
            if (!there[r]) continue;
            w.load(t[r], at<IN>(table.data, (uint64_t)row[r] * table.stride), dim);
        }
#pragma unroll
        for (uint32_t r = 0; r < kLookups; ++r) {
            if (p + r * per >= ids.count) break;
            float v[V];
            t[r].get(v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = there[r] ? v[i] * scale : 0.0f;
            w.template store_once<OUT>(at<OUT>(out.data, (p + r * per) * out.stride), v, dim);
        }
    }
}

// ---- rows that become zero ----------------------------------------------------------------------------
// rows [first, end) are cleared, those that a position names (named[r] != 0) excepted; named == nullptr: all of them
struct ClearRows {
    RowMatrix out;
    const uint8_t* named;
    uint64_t first, end;
    uint32_t dim, shift;    // 1 << shift lanes hold a row or a slice of it
    uint32_t slices;
};
template <int OUT>
__device__ __forceinline__ void clear_rows(const ClearRows& c, uint32_t block, uint32_t blocks) {
    constexpr int V = OUT == kF32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & ((1u << c.shift) - 1u), per = blockDim.x >> c.shift;
    const float zero[V] = {};
    for (uint64_t row = c.first + (uint64_t)block * per + (threadIdx.x >> c.shift); row < c.end; row += (uint64_t)blocks * per) {
        if (c.named != nullptr && c.named[row] != 0u) continue;
        for (uint32_t s = 0; s < c.slices; ++s) {
            const uint32_t col = ((s << c.shift) + lane) * V;
            if (col < c.dim) Window<V>(col, c.dim).template store_once<OUT>(at<OUT>(c.out.data, row * c.out.stride), zero, c.dim);
        }
    }
}
__device__ __forceinline__ void clear_rows(const ClearRows& c, uint32_t block, uint32_t blocks) {
    if (c.first < c.end) with_dtype(c.out.dtype, [&](auto o) { clear_rows<o>(c, block, blocks); });
}

__global__ __launch_bounds__(kThreads) void clear_rows_kernel(const ClearRows c) { clear_rows(c, blockIdx.x, gridDim.x); }

// ---- the sort ------------------------------------------------------------------------------------------
// Least significant digit first.  Every workgroup owns a range of the positions; a pass counts each range's digits, and the
// scatter adds up the counts before its own (of smaller digits, and of equal ones in earlier ranges) by itself.  The sort of a
// batch is a handful of workgroups that wait for memory, so the launches clear rows of the table beside it.
constexpr uint32_t kSortThreads = 512, kSortWaves = kSortThreads / 64u, kSortItems = 1, kSortTile = kSortThreads * kSortItems;
// Every workgroup reads all ranges' counts: a range holds up to four tiles before there are more than kRanges of them.  (16384 positions
// of 1024 values in tiles of 512, 1024, 2048 and 4096: 44.5, 46.5, 51 and 60 us.)
constexpr uint32_t kRanges = 64, kMaxRanges = 256, kRangeTiles = 4;
constexpr uint32_t kMaxDigitBits = 10, kMaxDigits = 1u << kMaxDigitBits;

constexpr uint64_t kClearBeside = 50000000;   // bytes
constexpr uint32_t kClearBlocks = 2048;          // what the GPU holds, twice over

struct SortShape {
    uint32_t passes, bits, ranges;
    uint64_t range;                       // positions of one, a multiple of kSortTile
    uint64_t most_counts;                 // no fewer than ranges << bits, here and for fewer positions and rows
};
SortShape sort_shape(uint64_t tokens, uint64_t rows) {
    SortShape s;
    uint32_t all = 1;
    while ((rows >> all) != 0u) ++all;    // keys are 0 .. rows
    s.passes = (all + kMaxDigitBits - 1u) / kMaxDigitBits;
    s.bits = (all + s.passes - 1u) / s.passes;
    const uint64_t tiles = (tokens + kSortTile - 1u) / kSortTile;
    const uint64_t most = std::min<uint64_t>(kMaxRanges, std::max<uint64_t>(kRanges, tiles / kRangeTiles)), each = (tiles + most - 1u) / most;
    s.range = each * kSortTile;
    s.ranges = (uint32_t)((tokens + s.range - 1u) / s.range);
    s.most_counts = std::min(tiles, most) << std::min(all, kMaxDigitBits);
    return s;
}

// Long runs are listed by the chunk they begin in (two neighbours are not both one's): with one counter for all, 400 of them wait for
// each other (65536 positions of 64 values: the sums took 14.7 us instead of 11.5).
constexpr uint32_t kJoinLists = 64, kJoinLine = 16;   // counters, and words between them
inline uint64_t join_capacity(uint64_t chunks) { return (chunks / 2u + kJoinLists) / kJoinLists * kJoinLists; }

struct SortArgs {
    TokenIds ids;
    uint64_t rows;
    const uint32_t* keys;     // nullptr: the first pass, which reads the tokens
    const uint32_t* order;
    uint32_t* keys_out;
    uint32_t* order_out;
    uint32_t* counts;         // [ranges][1 << bits]
    uint4* named;             // first pass, where rows are cleared: [rows] bytes, zeroed by the count and set by the scatter
    uint32_t* join_counts;    // cleared by the first launch
    uint64_t range;
    uint32_t ranges, bits, shift;
};

template <bool WIDE>
__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, uint64_t i) {
    return a.keys != nullptr ? a.keys[i] : row_of<WIDE>(a.ids, i, a.rows, true);
}

// How many keys of digit d come before this lane's: those that counts[d] holds from before, and those of lower lanes.  Adds the wave's
// keys to `counts`, which is the wave's own.
template <class Count>
__device__ __forceinline__ uint32_t rank_in_wave(Count* counts, uint32_t d, uint32_t bits, bool valid) {
    uint64_t same = __builtin_amdgcn_ballot_w64(valid);
    for (uint32_t b = 0; b < bits; ++b) {
        const bool one = (d >> b) & 1u;
        const uint64_t ones = __builtin_amdgcn_ballot_w64(one);
        same &= one ? ones : ~ones;
    }
    const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
    uint32_t seen = 0;
    if (valid) seen = __hip_atomic_load(&counts[d], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
    __builtin_amdgcn_wave_barrier();   // a wave's LDS operations keep their order: all have read before one writes
    if (valid && below == 0u) __hip_atomic_store(&counts[d], (Count)(seen + (uint32_t)__builtin_popcountll(same)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
    __builtin_amdgcn_wave_barrier();
    return seen + below;
}

template <bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a, const ClearRows c) {
    __shared__ uint32_t s_count[kMaxDigits];
    const uint32_t digits = 1u << a.bits;
    if (a.keys == nullptr && blockIdx.x == 0u && threadIdx.x < kJoinLists) a.join_counts[threadIdx.x * kJoinLine] = 0u;
    if (a.named != nullptr) {
        const uint64_t all = (a.rows + 15u) / 16u;
        for (uint64_t i = (uint64_t)blockIdx.x * kSortThreads + threadIdx.x; i < all; i += (uint64_t)gridDim.x * kSortThreads) a.named[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (blockIdx.x >= a.ranges) {
        clear_rows(c, blockIdx.x - a.ranges, gridDim.x - a.ranges);
        return;
    }
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) s_count[d] = 0u;
    __syncthreads();
    const uint64_t first = (uint64_t)blockIdx.x * a.range, end = min(first + a.range, a.ids.count);
    for (uint64_t tile = first; tile < end; tile += kSortTile) {
        uint32_t key[kSortItems];
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            const uint64_t i = tile + j * kSortThreads + threadIdx.x;
            if (i < end) key[j] = sort_key<WIDE>(a, i);
        }
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            if (tile + j * kSortThreads + threadIdx.x < end) atomicAdd(&s_count[(key[j] >> a.shift) & (digits - 1u)], 1u);
        }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.counts[(uint64_t)blockIdx.x * digits + d] = s_count[d];
}

template <bool WIDE>
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const SortArgs a, const ClearRows c) {
    __shared__ uint32_t s_next[kMaxDigits];                             // where the next key of a digit goes
    __shared__ uint32_t s_wave[kSortWaves][kMaxDigits];
    __shared__ uint32_t s_total[kSortWaves];
    if (blockIdx.x >= a.ranges) {
        clear_rows(c, blockIdx.x - a.ranges, gridDim.x - a.ranges);
        return;
    }
    const uint32_t digits = 1u << a.bits, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;

    const uint64_t first = (uint64_t)blockIdx.x * a.range, end = min(first + a.range, a.ids.count);
    const uint32_t mine = wave * (64u * kSortItems) + lane;   // a wave's keys are consecutive, 64 at a time
    uint32_t key[kSortItems], from[kSortItems];
    const auto load = [&](uint64_t tile) {
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            const uint64_t i = tile + mine + j * 64u;
            key[j] = i < end ? sort_key<WIDE>(a, i) : 0u;
            from[j] = i < end && a.order != nullptr ? a.order[i] : (uint32_t)i;
        }
    };
    load(first);   // on their way while the counts are added up

    // the keys of a digit in all ranges (s_wave[0]), and in the earlier ones (s_next); the threads share the ranges out where digits are
    // fewer.  (Counted here by every workgroup from all positions, without launches of their own: 66 -> 79 us for 16384 positions.)
    for (uint32_t d = tid; d < digits; d += kSortThreads) s_next[d] = s_wave[0][d] = 0u;
    __syncthreads();
    {
        const uint32_t shares = digits < kSortThreads ? kSortThreads / digits : 1u;
        for (uint32_t d0 = tid; d0 < digits * shares; d0 += kSortThreads) {
            const uint32_t d = d0 & (digits - 1u), share = d0 >> a.bits;
            uint32_t before = 0, all = 0;
            constexpr uint32_t kAhead = 16;
            for (uint32_t r0 = share; r0 < a.ranges; r0 += kAhead * shares) {
                uint32_t n[kAhead];
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    const uint32_t r = r0 + j * shares;
                    n[j] = r < a.ranges ? a.counts[(uint64_t)r * digits + d] : 0u;
                }
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    all += n[j];
                    before += r0 + j * shares < blockIdx.x ? n[j] : 0u;
                }
            }
            atomicAdd(&s_next[d], before);
            atomicAdd(&s_wave[0][d], all);
        }
    }
    __syncthreads();
    // the keys of smaller digits: every thread adds up consecutive digits
    const uint32_t per = (digits + kSortThreads - 1u) / kSortThreads;   // 1 or 2
    uint32_t own = 0;
    for (uint32_t j = 0; j < per; ++j) own += tid * per + j < digits ? s_wave[0][tid * per + j] : 0u;
    uint32_t upto = own;
#pragma unroll
    for (uint32_t m = 1; m < 64u; m <<= 1) {
        const uint32_t other = __shfl_up(upto, m, 64);
        if (lane >= m) upto += other;
    }
    if (lane == 63u) s_total[wave] = upto;
    __syncthreads();
    uint32_t at = upto - own;
    for (uint32_t w = 0; w < wave; ++w) at += s_total[w];
    for (uint32_t j = 0; j < per; ++j) {
        const uint32_t d = tid * per + j;
        if (d >= digits) break;
        s_next[d] += at;
        at += s_wave[0][d];
    }

    for (uint64_t tile = first; tile < end; tile += kSortTile) {
        uint32_t rank[kSortItems];
        __syncthreads();
        for (uint32_t d = lane; d < digits; d += 64u) s_wave[wave][d] = 0u;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            rank[j] = rank_in_wave(s_wave[wave], (key[j] >> a.shift) & (digits - 1u), a.bits, tile + mine + j * 64u < end);
        }
        __syncthreads();
        for (uint32_t d = tid; d < digits; d += kSortThreads) {
            uint32_t next = s_next[d];
#pragma unroll
            for (uint32_t w = 0; w < kSortWaves; ++w) {
                const uint32_t n = s_wave[w][d];
                s_wave[w][d] = next;
                next += n;
            }
            s_next[d] = next;
        }
        __syncthreads();
#pragma unroll
        for (uint32_t j = 0; j < kSortItems; ++j) {
            if (tile + mine + j * 64u >= end) continue;
            const uint32_t to = s_wave[wave][(key[j] >> a.shift) & (digits - 1u)] + rank[j];
            a.keys_out[to] = key[j];
            a.order_out[to] = from[j];
            if (a.named != nullptr && key[j] < a.rows) reinterpret_cast<uint8_t*>(a.named)[key[j]] = 1u;
        }
        load(tile + kSortTile);
    }
}

// Batches that a workgroup holds are sorted by one launch: kBuckets workgroups read all positions, and each keeps those of its bucket, a
// row's remainder, and sorts them by the quotient in LDS.  Where its bucket begins is the number of positions of the buckets before, which
// it sees on the way.  So no workgroup waits for another, and the chain of count and scatter launches, each of which mostly waits for
// memory and for the one before it, is gone.  Rows come out grouped, not in order, and positions that add to none last, which is all that
// the sums ask for.  (The gradient of 5000 positions of 64 values, those launches and this one: 26 and 20.5 us, of which this 7.2; 12000 33.5
// and 23.8; 16384 of 1024 44 and 39; with 206 MB of rows cleared 54 and 51.5.)  Digits of 8 bits: the LDS of two workgroups fits a CU, so
// that rows are cleared beside.
constexpr uint32_t kOneThreads = 1024, kOneWaves = kOneThreads / 64u, kOneItems = 16, kOneTokens = kOneThreads * kOneItems;
constexpr uint32_t kBuckets = 256, kOneBits = 8, kOneDigits = 1u << kOneBits, kOneNamed = 1024;   // kOneNamed: quotients that have a flag in LDS
constexpr uint32_t kPositionBits = 14;   // of an entry, whose other bits are the quotient
static_assert(kOneNamed == kOneThreads, "a lane writes a flag");
static_assert(kOneTokens <= 1u << kPositionBits, "a position does not fit an entry");
bool one_sort(uint64_t tokens, uint64_t rows) { return tokens <= kOneTokens && (rows + kBuckets - 1u) / kBuckets < 1u << (32u - kPositionBits); }

// Buckets of up to so many positions are sorted by counting the smaller entries of each: 64 compared by one ballot.  (5000 positions of which
// one row has 400: the sort takes 11 us where 512 are compared, 7.2 where 64, 128 or 192 are, 8.7 with digits alone.)
constexpr uint32_t kOneCompared = 128;

// none: the quotient behind the rows', by which the last bucket sorts the positions that add to no row; bits, passes: of the quotients
template <bool WIDE, uint32_t ITEMS>
__global__ __launch_bounds__(kOneThreads) void sort_buckets_kernel(const SortArgs a, const ClearRows c, const uint32_t none, const uint32_t passes) {
    __shared__ uint32_t s_entry[ITEMS * kOneThreads];
    __shared__ uint16_t s_wave[kOneWaves][kOneDigits];
    __shared__ uint32_t s_mine[kOneWaves], s_below[kOneWaves], s_total[kOneWaves];
    __shared__ uint8_t s_named[kOneNamed];
    if (blockIdx.x >= kBuckets) {
        clear_rows(c, blockIdx.x - kBuckets, gridDim.x - kBuckets);
        return;
    }
    const uint32_t tid = threadIdx.x, lane = tid & 63u, all = (uint32_t)a.ids.count, rows = (uint32_t)a.rows, bucket = blockIdx.x;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const auto below_lane = [](uint64_t m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u)); };
    if (bucket == 0u && tid < kJoinLists) a.join_counts[tid * kJoinLine] = 0u;
    s_named[tid] = 0u;
    uint32_t count = 0, base = 0;
    {
        const uint32_t items = (all + kOneThreads - 1u) / kOneThreads, first = wave * 64u * items + lane;   // a wave's positions are consecutive
        uint32_t key[ITEMS];
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) key[j] = row_of<WIDE>(a.ids, min(first + j * 64u, all - 1u), rows, true);
        uint64_t own[ITEMS];
        uint32_t mine = 0, below = 0;
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            const bool valid = j < items && first + j * 64u < all;
            const uint32_t of = key[j] < rows ? key[j] % kBuckets : kBuckets - 1u;
            own[j] = __builtin_amdgcn_ballot_w64(valid && of == bucket);
            mine += (uint32_t)__builtin_popcountll(own[j]);
            below += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(valid && of < bucket));
        }
        if (lane == 0u) {
            s_mine[wave] = mine;
            s_below[wave] = below;
        }
        __syncthreads();
        uint32_t to = 0;
#pragma unroll
        for (uint32_t w = 0; w < kOneWaves; ++w) {
            if (w == wave) to = count;
            count += s_mine[w];
            base += s_below[w];
        }
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            if ((own[j] >> lane) & 1u) {
                const uint32_t quotient = key[j] < rows ? key[j] / kBuckets : none;
                s_entry[to + below_lane(own[j])] = quotient << kPositionBits | (first + j * 64u);
                if (quotient < kOneNamed) s_named[quotient] = 1u;
            }
            to += (uint32_t)__builtin_popcountll(own[j]);
        }
        __syncthreads();
    }
    if (a.named != nullptr) {
        const uint32_t row = tid * kBuckets + bucket;
        if (tid < none && row < rows) reinterpret_cast<uint8_t*>(a.named)[row] = s_named[tid];
    }
    const auto put = [&](uint32_t to, uint32_t entry) {
        const uint32_t quotient = entry >> kPositionBits;
        a.keys_out[base + to] = quotient == none ? rows : quotient * kBuckets + bucket;
        a.order_out[base + to] = entry & ((1u << kPositionBits) - 1u);
    };
    if (count <= kOneCompared) {
        uint32_t other[kOneCompared / 64u];
#pragma unroll
        for (uint32_t j = 0; j < kOneCompared / 64u; ++j) other[j] = j * 64u + lane < count ? s_entry[j * 64u + lane] : ~0u;
        for (uint32_t i = wave; i < count; i += kOneWaves) {
            const uint32_t entry = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_entry[i]);
            uint32_t to = 0;
#pragma unroll
            for (uint32_t j = 0; j < kOneCompared / 64u; ++j) {
                if (j * 64u < count) to += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(other[j] < entry));
            }
            if (lane == 0u) put(to, entry);
        }
        return;
    }
    const uint32_t digits = 1u << a.bits, items = (count + kOneThreads - 1u) / kOneThreads, first = wave * 64u * items + lane;
    uint32_t entry[ITEMS], rank[ITEMS];
    for (uint32_t pass = 0; pass < passes; ++pass) {
        const uint32_t shift = kPositionBits + pass * a.bits;
        for (uint32_t d = lane; d < digits; d += 64u) s_wave[wave][d] = 0u;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            if (j >= items) break;
            const uint32_t i = first + j * 64u;
            entry[j] = i < count ? s_entry[i] : 0u;
            rank[j] = rank_in_wave(s_wave[wave], (entry[j] >> shift) & (digits - 1u), a.bits, i < count);
        }
        __syncthreads();
        uint32_t total = 0;   // of digit tid
        if (tid < digits) {
#pragma unroll
            for (uint32_t w = 0; w < kOneWaves; ++w) {
                const uint32_t n = s_wave[w][tid];
                s_wave[w][tid] = (uint16_t)total;
                total += n;
            }
        }
        uint32_t upto = total;
#pragma unroll
        for (uint32_t m = 1; m < 64u; m <<= 1) {
            const uint32_t before = __shfl_up(upto, m, 64);
            if (lane >= m) upto += before;
        }
        if (lane == 63u) s_total[wave] = upto;
        __syncthreads();
        uint32_t before = upto - total;
        for (uint32_t w = 0; w < wave; ++w) before += s_total[w];
        if (tid < digits) {
#pragma unroll
            for (uint32_t w = 0; w < kOneWaves; ++w) s_wave[w][tid] = (uint16_t)(s_wave[w][tid] + before);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            if (j >= items) break;
            if (first + j * 64u >= count) continue;
            const uint32_t to = s_wave[wave][(entry[j] >> shift) & (digits - 1u)] + rank[j];
            if (pass + 1u < passes) s_entry[to] = entry[j];
            else put(to, entry[j]);
        }
        __syncthreads();
    }
}

// ---- a few positions ------------------------------------------------------------------------------------
// Without a sort: every workgroup finds the positions of its position's row among all of them, a quarter a wave, and adds up their
// slice of grad_out where its own is the first.  One launch, whose work is the square of the positions for every slice of 256 values.
// kFewWork: this is faster than sort, sums and joins, or level, for rows of several slices up to half of it and for rows of one slice up to
// all of it, but for 250 values and rows to clear; above half, rows of several slices take up to 45 % longer.  (Half-precision rows added to
// fp32 ones, positions x values, this and those: 500 x 512 4.2 and 14.6 us; 1000 x 1000 8.6 and 16.0; 2000 x 64 8.4 and 18.7; 2000 x 500 11.4
// and 17.6; 3300 x 250 16.1 and 19.2; 4000 x 16 18.3 and 23.2; 4000 x 250 18.8 and 19.5; 1700 x 1000 17.0 and 17.8; 2600 x 500 20.8 and 18.4;
// 2000 x 1000 20.4 and 18.7; 1200 x 2500 26.5 and 18.3.  With 20000 fp32 rows cleared beside: 1000 x 1000 23.0 and 25.2; 2000 x 500 17.9 and 20.4;
// 4000 x 250 22.7 and 19.7; 2000 x 1000 32.4 and 27.1.)  The slices are counted as fp32 values have them; half precision on both sides has half
// as many (with 20000 rows cleared, 2000 x 1000 17.8 and 21.3; 2600 x 500 15.7 and 19.8).
constexpr uint32_t kFewTokens = 4096, kFewSum = 8, kFewRows = 1024;
constexpr uint64_t kFewWork = 16000000;
// Few rows of the table have long runs, which one workgroup adds up (2000 positions of 64 values in 4 rows: 29 us against 16).  In a larger
// table a row that most positions name is not foreseen (4000 positions of 250 values, all of one row: 128 us against 31, half of them 60
// against 25; 1000 positions 30 and 17.6 against 20 and 19).
constexpr uint32_t kFewRun = 256;   // positions of a row, on average
bool few_positions(uint64_t tokens, uint32_t dim, uint64_t rows) {
    return tokens <= kFewTokens && tokens <= kFewRun * rows && tokens * tokens * ((dim + 255u) / 256u) <= kFewWork;
}
struct FewArgs {
    TokenIds ids;
    RowMatrix grad, out;
    uint32_t dim, slices;    // a wave holds a slice of a row
    uint32_t sums;           // workgroups that add up; the others clear clear_rows rows each
    uint32_t clear_rows, clear_shift, clear_slices;
    float scale;
    bool accumulate;
};
__device__ __forceinline__ uint32_t few_row(const TokenIds& t, uint32_t i, uint32_t rows) {
    return t.wide ? row_of<true>(t, i, rows, true) : row_of<false>(t, i, rows, true);
}
// ITEMS: positions that a lane searches at most (1000 positions of 1000 values, 8 and 4: 10.7 and 8.9 us; 512 of 4096, 4 and 2: 12.9 and 11.3)
template <int IN, int OUT, uint32_t ITEMS>
__global__ __launch_bounds__(kThreads) void sum_few_kernel(const FewArgs a) {
    constexpr int V = values_of(IN, OUT);
    constexpr uint32_t kWaves = kThreads / 64u;
    __shared__ uint16_t s_list[ITEMS * kThreads];
    __shared__ uint32_t s_found[kWaves];
    __shared__ float s_sum[kWaves - 1u][64][V];
    __shared__ uint8_t s_named[kFewRows];
    const uint32_t count = (uint32_t)a.ids.count, rows = (uint32_t)a.out.rows, tid = threadIdx.x, lane = tid & 63u;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const uint32_t items = (count + kThreads - 1u) / kThreads, first = wave * 64u * items;   // a wave's positions are consecutive
    uint32_t key[ITEMS];
#pragma unroll
    for (uint32_t j = 0; j < ITEMS; ++j) {
        const uint32_t at = first + j * 64u + lane;
        key[j] = j < items && at < count ? few_row(a.ids, at, rows) : ~0u;
    }
    if (blockIdx.x >= a.sums) {
        constexpr int VC = OUT == kF32 ? 4 : 8;
        const uint64_t from = (uint64_t)(blockIdx.x - a.sums) * a.clear_rows, end = min(from + a.clear_rows, a.out.rows);
        for (uint32_t i = tid; i < a.clear_rows; i += kThreads) s_named[i] = 0u;
        __syncthreads();
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            if (key[j] >= from && key[j] < end) s_named[key[j] - from] = 1u;
        }
        __syncthreads();
        const float zero[VC] = {};
        for (uint64_t row = from + (tid >> a.clear_shift); row < end; row += kThreads >> a.clear_shift) {
            if (s_named[row - from] != 0u) continue;
            for (uint32_t s = 0; s < a.clear_slices; ++s) {
                const uint32_t col = ((s << a.clear_shift) + (tid & ((1u << a.clear_shift) - 1u))) * VC;
                if (col < a.dim) Window<VC>(col, a.dim).template store_once<OUT>(at<OUT>(a.out.data, row * a.out.stride), zero, a.dim);
            }
        }
        return;
    }
    const uint32_t p = blockIdx.x / a.slices, col = ((blockIdx.x - p * a.slices) * 64u + lane) * V;
    const uint32_t k = (uint32_t)__builtin_amdgcn_readfirstlane((int)few_row(a.ids, p, rows));
    if (k >= rows) return;
    const bool in = col < a.dim;
    const Window<V> w(in ? col : 0u, a.dim);
    Pack<OUT, V> old;
    void* y = at<OUT>(a.out.data, (uint64_t)k * a.out.stride);
    if (a.accumulate && wave == 0u && in) w.load(old, y, a.dim);
    uint64_t match[ITEMS];
    uint32_t found = 0;
#pragma unroll
    for (uint32_t j = 0; j < ITEMS; ++j) {
        match[j] = __builtin_amdgcn_ballot_w64(key[j] == k);
        if (match[j] != 0u && first + j * 64u + (uint32_t)__builtin_ctzll(match[j]) < p) found |= 1u << 31;   // not the first position of its row
        found += (uint32_t)__builtin_popcountll(match[j]);
    }
    if (lane == 0u) s_found[wave] = found;
    __syncthreads();
    uint32_t before = 0;
    found = 0;
#pragma unroll
    for (uint32_t n = 0; n < kWaves; ++n) {
        if (n == wave) before = found;
        found += s_found[n] & ~(1u << 31);
        if (s_found[n] >> 31) return;
    }
#pragma unroll
    for (uint32_t j = 0; j < ITEMS; ++j) {
        const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(match[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)match[j], 0u));
        if (key[j] == k) s_list[before + below] = (uint16_t)(first + j * 64u + lane);
        before += (uint32_t)__builtin_popcountll(match[j]);
    }
    __syncthreads();
    float sum[V] = {};
    for (uint32_t n = wave; n < found; n += kWaves * kFewSum) {   // the waves take the positions in turn
        Pack<IN, V> t[kFewSum];
#pragma unroll
        for (uint32_t j = 0; j < kFewSum; ++j) {
            if (!in || n + j * kWaves >= found) break;
            w.load(t[j], at<IN>(a.grad.data, (uint64_t)s_list[n + j * kWaves] * a.grad.stride), a.dim);
        }
#pragma unroll
        for (uint32_t j = 0; j < kFewSum; ++j) {
            if (!in || n + j * kWaves >= found) break;
            float v[V];
            t[j].get(v);
#pragma unroll
            for (int l = 0; l < V; ++l) sum[l] += v[l];
        }
    }
    if (found > 1u) {
        if (wave > 0u) {
#pragma unroll
            for (int l = 0; l < V; ++l) s_sum[wave - 1u][lane][l] = sum[l];
        }
        __syncthreads();
    }
    if (wave > 0u || !in) return;
    for (uint32_t n = 1; n < min(found, kWaves); ++n) {
#pragma unroll
        for (int l = 0; l < V; ++l) sum[l] += s_sum[n - 1u][lane][l];
    }
    float v[V];
    if (a.accumulate) {
        old.get(v);
#pragma unroll
        for (int l = 0; l < V; ++l) v[l] = __builtin_fmaf(a.scale, sum[l], v[l]);
        w.template store_own<OUT>(y, v, a.dim);
    } else {
#pragma unroll
        for (int l = 0; l < V; ++l) v[l] = a.scale * sum[l];
        w.template store_once<OUT>(y, v, a.dim);
    }
}

// ---- the sums ------------------------------------------------------------------------------------------
// The sorted positions are cut into chunks, and the lanes of a chunk add up its runs, eight rows of grad_out in flight.  A run
// that starts in a chunk and ends in the next one is added up by the chunk it starts in; one that goes on into the chunk after
// that is long: each of its chunks leaves a partial sum, which join_runs_kernel adds up in the order of the chunks.  So a row
// of the table that half a batch names is read by as many workgroups as any other half, and every chunk can tell from the
// keys around it which of its runs are whose.  The keys and the order around a workgroup's chunks are in LDS before the first
// row is asked for: loaded where they are needed, each of them waits for the loads and stores before it (131072 tokens of
// 4096 half-precision values into fp32: 457 -> 386 us; with 16-byte stores of whole lines and streaming loads 326, 5.1 TB/s of
// the rows read and written).
constexpr uint32_t kRows = 8;         // in flight
constexpr uint32_t kMostChunk = 64, kMostPositions = 2048;   // of a chunk, and of a workgroup's chunks together
constexpr uint32_t kShortestChunk = kMostPositions / kThreads;

struct SumArgs {
    const uint32_t *keys, *order;
    uint64_t count;                       // positions
    RowMatrix grad, out;
    float* partials;                      // [chunks][2][width]: of the long run that a chunk begins in, and of the one that begins in it
    uint2* joins;                         // the long runs, in kJoinLists lists: the chunk that one begins in, and its partial sums
    uint32_t* join_counts;                // of the lists, kJoinLine apart
    uint32_t dim, width, chunk;           // width: dim, rounded up to 8
    uint32_t shift, slices;               // 1 << shift lanes hold a row, or one of its slices
    float scale;
    bool accumulate;
};

// old: what the row held, where that is added to
template <bool ACCUMULATE, int OUT, int V>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, const Window<V>& w, const float (&sum)[V], const Pack<OUT, V>& old) {
    void* y = at<OUT>(a.out.data, (uint64_t)row * a.out.stride);
    float v[V];
    if constexpr (ACCUMULATE) {
        old.get(v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(a.scale, sum[i], v[i]);
        w.template store_own<OUT>(y, v, a.dim);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = a.scale * sum[i];
        w.template store_once<OUT>(y, v, a.dim);
    }
}

// Puts the long runs that begin in the wave's chunks down for join_runs_kernel: lanes with `begins`, each for a run of key k in `chunk`.
// A run ends with the last chunk that begins in it; the search goes on here, where other workgroups have work to do meanwhile.
// Call with every lane of the wave active.
__device__ __forceinline__ void list_runs(const SumArgs& a, bool begins, uint32_t chunk, uint32_t k) {
    const uint32_t lane = threadIdx.x & 63u;
    for (uint64_t left = __builtin_amdgcn_ballot_w64(begins); left != 0u; left &= left - 1u) {
        const int from = __builtin_ctzll(left);
        const uint32_t c = (uint32_t)__builtin_amdgcn_readlane((int)chunk, from), key = (uint32_t)__builtin_amdgcn_readlane((int)k, from);
        uint64_t low = 2, high = (a.count - 1u) / a.chunk - c + 1u;   // chunk c + low - 1 begins in the run, chunk c + high does not
        for (uint64_t step = 1; low < high; step = (high - low + 63u) / 64u) {   // 64 at a time, the nearest first, which are all of most runs
            const uint64_t probe = low + lane * step;
            const bool in = probe < high && a.keys[(c + probe) * a.chunk] == key;
            const uint32_t seen = (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in));
            if (seen < 64u) high = min(high, low + seen * step);
            if (seen > 0u) low += (seen - 1u) * step + 1u;
        }
        if (lane == 0u) {
            const uint32_t list = (c >> 1) % kJoinLists, n = atomicAdd(a.join_counts + list * kJoinLine, 1u);
            a.joins[(uint64_t)n * kJoinLists + list] = make_uint2(c, (uint32_t)low);
        }
    }
}

// The chunks of a workgroup, in one slice.  UNIFORM: a wave's lanes all belong to one chunk.
// ACCUMULATE: the old row of a run is on its way with the run's first row.  (Asked for when the run has been added up, the gradient of
// 300000 rows of 256 values added to fp32 rows took 111 us instead of 101; of 16384 of 1024 values 45 and 43.8.)
template <int IN, int OUT, bool UNIFORM, bool ACCUMULATE>
__device__ __forceinline__ void sum_chunks(const SumArgs& a, const uint64_t block, const uint32_t slice, uint32_t* s_key, uint32_t* s_order) {
    constexpr int V = values_of(IN, OUT);
    const uint32_t lane = threadIdx.x & ((1u << a.shift) - 1u), per = kThreads >> a.shift, col = ((slice << a.shift) + lane) * V;
    const uint32_t rows = (uint32_t)a.out.rows;
    const uint64_t base = block * per * a.chunk;             // the workgroup's first position; s_key begins chunk + 1 before it
    const uint32_t before = a.chunk + 1u;
    for (uint32_t i = threadIdx.x; i < per * a.chunk + 2u * a.chunk + 2u; i += kThreads) {
        const uint64_t p = base + i - before;                // wraps far beyond the last position
        s_key[i] = p < a.count ? a.keys[p] : ~0u;            // no row and no token's key
    }
    for (uint32_t i = threadIdx.x; i < per * a.chunk + a.chunk; i += kThreads) s_order[i] = base + i < a.count ? a.order[base + i] : 0u;
    __syncthreads();
    uint32_t team = threadIdx.x >> a.shift;
    if constexpr (UNIFORM) team = (uint32_t)__builtin_amdgcn_readfirstlane((int)team);
    const auto scalar = [](uint32_t x) { return UNIFORM ? (uint32_t)__builtin_amdgcn_readfirstlane((int)x) : x; };
    const auto key = [&](uint32_t i) { return scalar(s_key[i + before]); };   // i: from the workgroup's first position
    // does the run of key k, which goes on across the beginning i of a chunk, reach beyond a chunk on one of its sides?
    const auto is_long = [&](uint32_t i, uint32_t k) { return key(i - a.chunk - 1u) == k || key(i + a.chunk) == k; };

    const uint32_t start = team * a.chunk, end = start + a.chunk;
    uint32_t cur = key(start);
    const bool continues = key(start - 1u) == cur, head = continues && is_long(start, cur);
    const uint32_t last = key(end - 1u);
    const bool tail = last < rows && key(end) == last && is_long(end, last);
    const uint64_t chunk = block * per + team;
    list_runs(a, slice == 0u && lane == 0u && tail && !(continues && cur == last), (uint32_t)chunk, last);
    if (cur >= rows || col >= a.dim) return;               // such keys are the last: no position from here on adds to a row
    uint32_t i = start, stop = end;
    if (continues && !head) {                              // the chunk before this one adds it up
        while (i < end && key(i) == cur) ++i;
        if (i == end || key(i) >= rows) return;
        cur = key(i);
    }
    if (last >= rows) {
        while (key(stop - 1u) >= rows) --stop;
    } else if (!tail) {
        while (key(stop) == last) ++stop;                  // less than a chunk: the run is not long
    }
    const Window<V> w(col, a.dim);
    float sum[V] = {};
    uint32_t run = head ? 0u : ~0u;                        // the slot of the run's partial sum; ~0u: the run is whole
    Pack<OUT, V> old = {};
    bool first = true;                                     // no row has been asked for
    const auto finish = [&] {
        if (run == ~0u) {
            write_row<ACCUMULATE, OUT, V>(a, cur, w, sum, old);
            return;
        }
        Pack<kF32, V> o;
        o.set(sum);
        o.store(a.partials + (2u * chunk + run) * a.width + w.at);
    };
    for (; i < stop; i += kRows) {
        Pack<IN, V> t[kRows];
#pragma unroll
        for (uint32_t j = 0; j < kRows; ++j) {             // past the end: the last row again
            const uint32_t from = scalar(s_order[min(i + j, stop - 1u)]);
            w.load_once(t[j], at<IN>(a.grad.data, (uint64_t)from * a.grad.stride), a.dim);
        }
        Pack<OUT, V> next[ACCUMULATE ? kRows : 1u];
        if constexpr (ACCUMULATE) {
#pragma unroll
            for (uint32_t j = 0; j < kRows; ++j) {
                const uint32_t k = key(min(i + j, stop - 1u));
                if (j == 0u ? first || k != cur : k != key(min(i + j - 1u, stop - 1u))) {
                    w.load(next[j], at<OUT>(a.out.data, (uint64_t)k * a.out.stride), a.dim);
                }
            }
            if (first) old = next[0];
            first = false;
        }
#pragma unroll
        for (uint32_t j = 0; j < kRows; ++j) {
            if (i + j >= stop) break;
            const uint32_t k = key(i + j);
            if (k != cur) {
                finish();
                cur = k;
                run = ~0u;
                if constexpr (ACCUMULATE) old = next[j];
#pragma unroll
                for (int l = 0; l < V; ++l) sum[l] = 0.0f;
            }
            float v[V];
            t[j].get(v);
#pragma unroll
            for (int l = 0; l < V; ++l) sum[l] += v[l];
        }
    }
    if (tail && run == ~0u) run = 1u;
    finish();
}
template <int IN, int OUT, bool UNIFORM, bool ACCUMULATE>
__global__ __launch_bounds__(kThreads) void sum_runs_kernel(const SumArgs a, const ClearRows c, const uint32_t sums) {
    if (blockIdx.x >= sums) {
        if constexpr (!ACCUMULATE) clear_rows<OUT>(c, blockIdx.x - sums, gridDim.x - sums);
        return;
    }
    __shared__ uint32_t s_key[kMostPositions + 2u * kMostChunk + 2u], s_order[kMostPositions + kMostChunk];
    const uint32_t first = blockIdx.x / a.slices, slice = blockIdx.x - first * a.slices;
    const uint64_t blocks = (a.count + (uint64_t)(kThreads >> a.shift) * a.chunk - 1u) / ((kThreads >> a.shift) * a.chunk);
    for (uint64_t block = first; block < blocks; block += sums / a.slices) {
        sum_chunks<IN, OUT, UNIFORM, ACCUMULATE>(a, block, slice, s_key, s_order);
        __syncthreads();
    }
}

// The partial sums of a long run: `1 << join_shift` lanes hold one (or a slice of one), four values each; they take them in turn, add up
// theirs in order, and one of them adds up all.
constexpr uint32_t kJoinThreads = 1024, kJoinBlocks = 512;
template <int OUT>
__global__ __launch_bounds__(kJoinThreads) void join_runs_kernel(const SumArgs a, const uint32_t shift) {
    __shared__ float s_sum[kJoinThreads][4];
    const uint32_t teams = kJoinThreads >> shift, team = threadIdx.x >> shift, col = ((blockIdx.y << shift) + (threadIdx.x & ((1u << shift) - 1u))) * 4u;
    const uint32_t list = blockIdx.x % kJoinLists, joins = a.join_counts[list * kJoinLine];
    for (uint32_t n = blockIdx.x / kJoinLists; n < joins; n += gridDim.x / kJoinLists) {
        const uint2 join = a.joins[(uint64_t)n * kJoinLists + list];
        const uint64_t c = join.x;
        const uint32_t parts = join.y;                                // slot 1 of c, slot 0 of c + 1 .. c + parts - 1
        const uint32_t k = a.keys[(c + 1u) * a.chunk];
        float sum[4] = {};
        if (col < a.width) {
            constexpr uint32_t kAhead = 8;
            for (uint32_t p = team; p < parts; p += kAhead * teams) {
                Pack<kF32, 4> t[kAhead];
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    const uint32_t part = min(p + j * teams, parts - 1u);
                    t[j].load(a.partials + (2u * (c + part) + (part == 0u ? 1u : 0u)) * a.width + col);
                }
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    if (p + j * teams >= parts) break;
                    float v[4];
                    t[j].get(v);
#pragma unroll
                    for (int l = 0; l < 4; ++l) sum[l] += v[l];
                }
            }
        }
        __syncthreads();                                              // the run before this one has been added up
#pragma unroll
        for (int l = 0; l < 4; ++l) s_sum[threadIdx.x][l] = sum[l];
        __syncthreads();
        if (team == 0u && col < a.dim) {
            for (uint32_t other = 1; other < min(teams, parts); ++other) {
#pragma unroll
                for (int l = 0; l < 4; ++l) sum[l] += s_sum[(other << shift) + threadIdx.x][l];
            }
            // from four values at `col` to a window of the row
            const Window<4> w(col, a.dim);
            void* y = at<OUT>(a.out.data, (uint64_t)k * a.out.stride);
#pragma unroll
            for (int l = 0; l < 4; ++l) {
                if (w.skip != 0u || w.narrow) {
                    if (col + l < a.dim) store_one<OUT>(y, col + l, a.accumulate ? __builtin_fmaf(a.scale, sum[l], load_one<OUT>(y, col + l)) : a.scale * sum[l]);
                }
            }
            if (w.skip == 0u && !w.narrow) {
                Pack<OUT, 4> old = {};
                if (a.accumulate) w.load(old, y, a.dim);
                if (a.accumulate) write_row<true, OUT, 4>(a, k, w, sum, old);
                else write_row<false, OUT, 4>(a, k, w, sum, old);
            }
        }
    }
}

// How `rows` rows are shared out: 1 << shift lanes hold a row, or one of `slices` slices of it; the workgroups take rows in turn
// where a launch, which holds less than 2^32 lanes, has no workgroup for each.
struct RowShape {
    uint32_t shift, slices, blocks;
};
constexpr uint64_t kMaxBlocks = 1u << 23;
RowShape row_shape(uint64_t rows, uint32_t dim, uint32_t v) {
    RowShape s = {};
    while ((1u << s.shift) < kThreads && (1u << s.shift) * v < dim) ++s.shift;
    s.slices = (dim + (v << s.shift) - 1u) / (v << s.shift);
    const uint64_t per = kThreads >> s.shift, most = std::max<uint64_t>(1, kMaxBlocks / s.slices);
    s.blocks = (uint32_t)std::min<uint64_t>((rows + per - 1u) / per, most) * s.slices;
    return s;
}

// Positions of a chunk: as many as leave 4096 waves, and as many as leave 1024 where there are more than 2048 chunks, whose partial sums
// a long run's join waits for; no more than LDS holds of a workgroup's.  (65536 positions of 435 values, 8 and 32: 72 and 68 us; of 64
// values, which leave 256 waves with chunks of 32: 46 and 53; 131072 of 4096 values, 16, 32 and 64: 698, 654 and 632.)  The same for all
// types, which the size of the workspace does not depend on.
uint32_t chunk_of(uint64_t tokens, uint32_t dim) {
    const RowShape g = row_shape(1, dim, 8u);
    const uint32_t per = kThreads >> g.shift;                       // most chunks of a workgroup: 8 values a lane
    const uint64_t waves = tokens * g.slices * (kThreads / 64u) / per;   // of chunks of one position
    uint32_t chunk = kShortestChunk;
    while (chunk < kMostChunk && per * chunk < kMostPositions &&
           (waves / (2u * chunk) >= 4096u || (waves / (2u * chunk) >= 1024u && tokens / chunk > 2048u))) {
        chunk *= 2u;
    }
    return chunk;
}

// Floats of one slot of all chunks' partial sums, for so many positions or fewer and rows of `width` values or less: longer chunks, of which
// there are fewer, make the need itself fall where a batch grows.  chunk_of stops at one of three: chunks of kMostChunk; chunks of which a
// workgroup's hold kMostPositions (2048 / chunk of them, each of 2048 values a workgroup's row at most: a float for every position); or fewer
// than 4096 waves from chunks twice as long, which leaves at most 2048 * 2048 values.
uint64_t most_partials(uint64_t tokens, uint64_t width) {
    const uint64_t most = std::max<uint64_t>({2048u * 2048u, (tokens + kMostChunk - 1u) / kMostChunk * width, tokens}) + width;
    return std::min((tokens + kShortestChunk - 1u) / kShortestChunk * width, most);
}

struct GradWorkspace {
    uint32_t *keys[2], *order[2], *counts, *named, *join_counts;
    uint2* joins;
    float* partials;
    size_t bytes;
};
// Every part is the larger the more positions, values and rows there are, so that a workspace serves all smaller batches.
GradWorkspace grad_workspace(void* base, uint64_t tokens, uint32_t dim, uint64_t rows) {
    GradWorkspace w = {};
    w.named = static_cast<uint32_t*>(base);
    w.bytes = (rows + 15u) & ~(uint64_t)15u;
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
    w.counts = take(s.most_counts);
    w.join_counts = take(kJoinLists * kJoinLine);
    w.joins = reinterpret_cast<uint2*>(take(2u * join_capacity((tokens + kShortestChunk - 1u) / kShortestChunk)));
    w.partials = reinterpret_cast<float*>(take(2u * most_partials(tokens, (dim + 7u) & ~7u)));
    return w;
}

}  // namespace

hipError_t launch_embedding(const RowMatrix& table, const TokenIds& ids, uint32_t dim, float scale, const RowMatrix& out, hipStream_t stream) {
    if (ids.count == 0) return hipSuccess;
    with_dtype(table.dtype, [&](auto in) {
        with_dtype(out.dtype, [&](auto o) {
            constexpr uint32_t v = values_of(in, o);
            const RowShape g = row_shape((ids.count + kLookups - 1u) / kLookups, dim, v);
            hipLaunchKernelGGL((ids.wide ? embedding_kernel<in, o, true> : embedding_kernel<in, o, false>), dim3(g.blocks), dim3(kThreads), 0, stream, table, ids,
                               dim, g.shift, g.slices, scale, out);
        });
    });
    return hipGetLastError();
}

bool embedding_grad_takes_workspace(uint64_t tokens, uint32_t dim, uint64_t rows) { return tokens != 0 && !few_positions(tokens, dim, rows); }
size_t embedding_grad_workspace(uint64_t tokens, uint32_t dim, uint64_t rows) {
    // a table of fewer rows is sorted
    if (!embedding_grad_takes_workspace(tokens, dim, rows)) rows = tokens == 0 ? 0 : (tokens - 1u) / kFewRun;
    return rows == 0 ? 0 : grad_workspace(nullptr, tokens, dim, rows).bytes;
}

hipError_t launch_embedding_grad(const RowMatrix& grad_out, const TokenIds& ids, uint32_t dim, float scale, const RowMatrix& table_grad,
                                 bool accumulate, void* workspace, hipStream_t stream) {
    ClearRows clear = {};
    clear.out = table_grad;
    clear.dim = dim;
    const auto clear_shape = [&](uint64_t rows) { return row_shape(rows, dim, table_grad.dtype == kF32 ? 4u : 8u); };
    clear.shift = clear_shape(1).shift;
    clear.slices = clear_shape(1).slices;
    if (ids.count == 0) {
        if (accumulate) return hipSuccess;
        clear.end = table_grad.rows;
        hipLaunchKernelGGL(clear_rows_kernel, dim3(clear_shape(clear.end).blocks / clear.slices), dim3(kThreads), 0, stream, clear);
        return hipGetLastError();
    }
    if (few_positions(ids.count, dim, table_grad.rows)) {
        FewArgs f = {};
        f.ids = ids;
        f.grad = grad_out;
        f.out = table_grad;
        f.dim = dim;
        f.scale = scale;
        f.accumulate = accumulate;
        f.clear_shift = clear.shift;
        f.clear_slices = clear.slices;
        // a workgroup clears 16 KB at least; 4096 workgroups, or as many as hold the rows
        const uint64_t row_bytes = (uint64_t)dim * bytes_of(table_grad.dtype);
        f.clear_rows = (uint32_t)std::min<uint64_t>(kFewRows, std::max<uint64_t>({1u, 16384u / row_bytes, (table_grad.rows + 4095u) / 4096u}));
        const uint32_t clears = accumulate ? 0u : (uint32_t)((table_grad.rows + f.clear_rows - 1u) / f.clear_rows);
        with_dtype(grad_out.dtype, [&](auto in) {
            with_dtype(table_grad.dtype, [&](auto o) {
                constexpr uint32_t width = 64u * values_of(in, o);
                f.slices = (dim + width - 1u) / width;
                f.sums = (uint32_t)ids.count * f.slices;
                const auto kernel = ids.count <= 4u * kThreads ? (ids.count <= 2u * kThreads ? sum_few_kernel<in, o, 2u> : sum_few_kernel<in, o, 4u>)
                                                               : (ids.count <= 8u * kThreads ? sum_few_kernel<in, o, 8u> : sum_few_kernel<in, o, 16u>);
                hipLaunchKernelGGL(kernel, dim3(f.sums + clears), dim3(kThreads), 0, stream, f);
            });
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
    a.join_counts = w.join_counts;
    // The rows to clear are shared out over the launches of the sort: to each but the last as much as takes about as long as the
    // launch does without, to the last all that is left.  Rows that are cleared before the names are known are cleared for
    // nothing where they are named, which the last rows of a vocabulary seldom are: from the last row on.
    uint64_t left = accumulate ? 0 : table_grad.rows;
    const uint64_t beside = std::max<uint64_t>(1, kClearBeside / ((uint64_t)dim * bytes_of(table_grad.dtype)));
    const auto share = [&](bool rest) {
        clear.end = left;
        left -= rest ? left : std::min(left, beside);
        clear.first = left;
        return (uint32_t)std::min<uint64_t>(kClearBlocks, clear.end - clear.first);
    };
    hipError_t e;
    const uint32_t none = (uint32_t)((table_grad.rows + kBuckets - 1u) / kBuckets);
    uint32_t none_bits = 1;
    while ((none >> none_bits) != 0u) ++none_bits;
    // Where rows are cleared and a bucket's have flags, the sums' launch clears those that no position names; otherwise the launches below do.
    const bool one = one_sort(ids.count, table_grad.rows) && (accumulate || none <= kOneNamed);
    if (one) {
        const uint32_t passes = (none_bits + kOneBits - 1u) / kOneBits;
        a.bits = (none_bits + passes - 1u) / passes;
        a.keys_out = w.keys[0];
        a.order_out = w.order[0];
        const bool small = ids.count <= kOneTokens / 2u;
        const auto kernel = ids.wide ? (small ? sort_buckets_kernel<true, kOneItems / 2u> : sort_buckets_kernel<true, kOneItems>)
                                     : (small ? sort_buckets_kernel<false, kOneItems / 2u> : sort_buckets_kernel<false, kOneItems>);
        // (50257 rows of 64 values: 20.5 us without any beside, 21.7 with)
        const uint32_t more = left > 2u * beside ? share(false) : 0u;
        hipLaunchKernelGGL(kernel, dim3(kBuckets + more), dim3(kOneThreads), 0, stream, a, clear, none, passes);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.keys = a.keys_out;
        a.order = a.order_out;
        clear.named = reinterpret_cast<const uint8_t*>(a.named);
    }
    for (uint32_t pass = 0; !one && pass < s.passes; ++pass) {
        a.keys_out = w.keys[pass & 1u];
        a.order_out = w.order[pass & 1u];
        a.shift = pass * s.bits;
        clear.named = pass == 0u ? nullptr : reinterpret_cast<const uint8_t*>(w.named);
        uint32_t more = share(false);
        if (a.named != nullptr) more = std::max<uint32_t>(more, (uint32_t)std::min<uint64_t>(kClearBlocks, a.rows / (32u * kSortThreads)));
        hipLaunchKernelGGL((ids.wide ? sort_count_kernel<true> : sort_count_kernel<false>), dim3(s.ranges + more), dim3(kSortThreads), 0, stream, a, clear);
        e = hipGetLastError();   // counts that nothing wrote would scatter anywhere
        if (e != hipSuccess) return e;
        more = share(pass + 1u == s.passes);
        hipLaunchKernelGGL((ids.wide ? sort_scatter_kernel<true> : sort_scatter_kernel<false>), dim3(s.ranges + more), dim3(kSortThreads), 0, stream, a, clear);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.keys = a.keys_out;
        a.order = a.order_out;
        a.named = nullptr;
    }
    SumArgs b = {};
    b.keys = a.keys;
    b.order = a.order;
    b.count = ids.count;
    b.grad = grad_out;
    b.out = table_grad;
    b.partials = w.partials;
    b.joins = w.joins;
    b.join_counts = w.join_counts;
    b.dim = dim;
    b.width = (dim + 7u) & ~7u;
    b.chunk = chunk_of(ids.count, dim);
    b.scale = scale;
    b.accumulate = accumulate;
    const uint64_t chunks = (ids.count + b.chunk - 1u) / b.chunk;
    clear.first = 0;
    clear.end = left;
    const uint32_t clears = left == 0u ? 0u : clear_shape(left).blocks / clear.slices;
    with_dtype(grad_out.dtype, [&](auto in) {
        with_dtype(table_grad.dtype, [&](auto o) {
            constexpr uint32_t v = values_of(in, o);
            const RowShape g = row_shape(chunks, dim, v);
            b.shift = g.shift;
            b.slices = g.slices;
            const auto kernel = accumulate ? (g.shift >= 6u ? sum_runs_kernel<in, o, true, true> : sum_runs_kernel<in, o, false, true>)
                                           : (g.shift >= 6u ? sum_runs_kernel<in, o, true, false> : sum_runs_kernel<in, o, false, false>);
            hipLaunchKernelGGL(kernel, dim3(g.blocks + clears), dim3(kThreads), 0, stream, b, clear, g.blocks);
        });
    });
    e = hipGetLastError();
    if (e != hipSuccess || chunks < 3u) return e;   // a long run touches three chunks
    with_dtype(table_grad.dtype, [&](auto o) {
        uint32_t shift = 0;
        while (shift < 6u && (4u << shift) < dim) ++shift;
        const uint32_t slice = 4u << shift;
        hipLaunchKernelGGL((join_runs_kernel<o>), dim3((uint32_t)std::min<uint64_t>(join_capacity(chunks), kJoinBlocks), (dim + slice - 1u) / slice), dim3(kJoinThreads), 0, stream, b, shift);
    });
    return hipGetLastError();
}

}  // namespace mqg
