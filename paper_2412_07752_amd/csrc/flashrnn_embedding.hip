// Embedding lookup and its gradient by sorted tokens (include/flashrnn.h).
//
// out_i = s E[tok_i];  dE[v] = s sum over the places i of v of dout_i, every sum in float32 and in an order that sizes and tokens alone decide, so that no result hangs on which workgroup comes first.  Both are bound by
// memory, the gradient of few places by its launches: 65536 places x 2048 columns in bf16 61 us (5.5 TB/s); gradient into 50304 words 157 us (4.3 TB/s: a sort of four launches takes 27 us of it, the sums
// and the zeros beside them 123, the pieces 8), 4096 places x 768 columns into 32000 words 25.9 us, 32 places of 64 columns 4.9 us.
//
// The gradient of few places (at most kFewPlaces) is one launch.  Beyond, it sorts the places by their word, stable, so that the places of a word stay in order: up to kSmall places by counting over all pairs,
// beyond by a radix sort, least significant digit first, of tiles of places.  The table's rows are filled with zeros by the workgroups that the sort leaves idle.  Then groups of lanes
// add up runs of consecutive sorted places and write the rows of the words that begin and end inside; what is left of a word at the ends of a run goes to the workspace, and a last kernel joins such pieces:
// in order where they are few, by several groups of lanes where a word goes on through kManyRuns runs and more.  Tokens outside the vocabulary sort behind all words.
#include "flashrnn_rows.h"

using namespace flashrnn;

namespace {

constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
// Places that are sorted by counting, the bits of their numbers, and those that a workgroup ranks.  Whole gradients of 80 columns among 32000 words: 4096 places 12.5 us by counting and 27.3 by tiles, 12288 places
// 24.8 and 29.2, 15360 places 33.2 and 30.1; of 768 columns 25.9 and 37.7, 40.5 and 42.1, 47.9 and 43.0.  Among 300 words, which tiles sort in one pass, counting is ahead up to some 8192 places
// (768 columns: 21.5 and 21.9; 12288 places 29.7 and 22.7).
constexpr int kSmall = 12288, kSmallBits = 14, kRanked = 16;
// Tiles of a larger sort, each of which adds up the counts of all: 300000 places of 64 columns 49.5 us, with 128 tiles 53.9 and with 512 as with 256; a million 66.3, 68.8, and with 512 90.
constexpr int kMaxTiles = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kTileRounds = 2;     // places per thread of a tile at a time
constexpr int kRows = 4;           // places that a group of lanes looks up at a time, where there are kManyWaves waves of places
constexpr uint64_t kManyWaves = 16384;
constexpr int kColumns = 4;        // columns a lane adds up: neighbours store whole cache lines of float32 (with eight, each store left every second 16 bytes out)
constexpr uint32_t kMinRun = 8, kMaxRun = 64;   // sorted places that a group of lanes adds up
constexpr size_t kFillWaves = 32768, kFillBytes = 8 << 10;   // waves that fill, at most; bytes of the table that a wave fills at a time
constexpr size_t kFillBesideSort = 64 << 20;                  // bytes of the table that are filled beside one launch of a sort of tiles
// With few places the table is filled beside the ranking, present words or not, but for so many bytes beside the sums, whose words are looked for among the sorted ones: 4096 places of 768 columns
// among 32000 words 25.4 us, all beside the ranking 26.5; 5000 of 1000 columns among 131072 words 112 and 115, and 132 where all but 64 MB are filled beside the sums.
constexpr size_t kFillBesideSums = 32 << 20;
constexpr size_t kFlagsPerBlock = 16 << 10, kFlagBlocks = 2048;

__device__ __forceinline__ uint32_t key_of(const void* tokens, bool index64, size_t i, uint32_t vocab) {
    const int64_t t = index64 ? ((const int64_t*)tokens)[i] : ((const int32_t*)tokens)[i];
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : vocab;
}

// A lane's columns: V of them from `at` on; the last ones of a row whose length is no multiple of V overlap the lane's before, by `skip` columns (V: another lane has them all).  NARROW:
// rows shorter than V, one lane's, value by value (decided when compiled: a branch around every load would wait for it).
template <int V, bool NARROW> struct Columns {
    int at, skip;
    __device__ __forceinline__ Columns(int chunk, int width) {
        const int last = width - V;
        if constexpr (NARROW) {
            at = 0;
            skip = chunk ? V : -last;   // (columns that there are not)
        } else {
            at = chunk * V > last ? last : chunk * V;
            skip = chunk * V >= width ? V : chunk * V - at;
        }
    }
    template <typename T> __device__ __forceinline__ Chunk<T, V> load(const T* row) const {
        Chunk<T, V> c;
        if constexpr (!NARROW) {
            c.load(row + at);
        } else {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < V - skip ? load_value(row + i) : 0.f;
            c.put(v);
        }
        return c;
    }
    template <typename T> __device__ __forceinline__ void store(T* row, const float (&v)[V], bool stream = false) const {
        if (skip == V) return;
        if constexpr (!NARROW) {
            Chunk<T, V> c;
            c.put(v);
            c.store(row + at, stream);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < V - skip) store_value(row + i, v[i]);
        }
    }
    // row += v: a column that two lanes hold is one's alone
    __device__ __forceinline__ void add(float* row, float (&v)[V]) const {
        if (skip == V) return;
        if (!NARROW && !skip) {
            Chunk<float, V> c;
            c.load(row + at);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += c.get(i);
            c.put(v);
            c.store(row + at);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (NARROW ? i < V - skip : i >= skip) row[at + i] += v[i];
        }
    }
};

// Lookup: groups of L lanes take V columns a lane of R places each, whose words and then whose rows are requested together (65536 x 2048 in bf16, stored through the caches: 78 us, with one place at a
// time 82).
struct Lookup {
    const void *table, *tokens;
    void* out;
    uint64_t n;
    uint32_t vocab, column_blocks;
    int width, index64, stream;
    float scale;
};
template <typename E, typename O, int L, int R, bool NARROW>
__global__ __launch_bounds__(kThreads) void embedding_fwd_kernel(Lookup q) {
    constexpr int V = sizeof(E) == 2 && sizeof(O) == 2 ? 8 : 4, kGroups = kThreads / L;
    const uint64_t step = (uint64_t)gridDim.x * kGroups, total = (q.n + R - 1) / R * q.column_blocks;
    for (uint64_t id = (uint64_t)blockIdx.x * kGroups + threadIdx.x / L; id < total; id += step) {
        const uint64_t part = id / q.column_blocks, first = part * R;
        const Columns<V, NARROW> col((int)(id - part * q.column_blocks) * L + threadIdx.x % L, q.width);
        uint32_t word[R];
#pragma unroll
        for (int u = 0; u < R; ++u) word[u] = key_of(q.tokens, q.index64, first + u < q.n ? first + u : q.n - 1, q.vocab);
        Chunk<E, V> row[R];
#pragma unroll
        for (int u = 0; u < R; ++u) row[u] = col.load((const E*)q.table + (size_t)(word[u] < q.vocab ? word[u] : 0) * q.width);   // (row 0 for places outside the vocabulary)
#pragma unroll
        for (int u = 0; u < R; ++u) {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = word[u] < q.vocab ? row[u].get(i) * q.scale : 0.f;
            if (first + u < q.n) col.store((O*)q.out + (size_t)(first + u) * q.width, v, q.stream);
        }
    }
}

// zeros for rows [begin, end) of the table, `each` (up to 64) at a time a wave, but for those that are `there`; neighbours in one go
struct Fill {
    float* table;
    const uint8_t* flags;
    const uint32_t* keys;
    uint32_t begin, end, each, n;
    int width;
};
// there(first, row, in): whether the lane's row, one of those from `first` on, is left alone (in: it is one of [begin, end))
template <int NT, typename There> __device__ __forceinline__ void fill_rows(const Fill& f, unsigned block, unsigned blocks, There there) {
    constexpr int kWaves = NT / kWave;
    const int lane = threadIdx.x & 63;
    Chunk<float, 4> zero;
    zero.clear();
    for (uint64_t first = f.begin + ((uint64_t)block * kWaves + threadIdx.x / kWave) * f.each; first < f.end; first += (uint64_t)blocks * kWaves * f.each) {
        const uint64_t row = first + lane;
        const bool in = (uint32_t)lane < f.each && row < f.end, stays = there((uint32_t)first, row, in);   // (by all lanes)
        uint64_t absent = __ballot(in && !stays);
        while (absent) {
            const int from = __builtin_ctzll(absent);
            const uint64_t rest = ~(absent >> from);
            const int count = rest ? __builtin_ctzll(rest) : kWave;
            float* at = f.table + (first + from) * f.width;
            const uint64_t n = (uint64_t)count * f.width;
            if (n < 4) {
                if ((uint32_t)lane < n) at[lane] = 0.f;
            } else {
                for (uint64_t i = (uint64_t)lane * 4; i < n; i += 4 * kWave) zero.store(at + (i + 4 <= n ? i : n - 4), true);
            }
            if (from + count >= kWave) break;
            absent &= ~0ull << (from + count);
        }
    }
}
// all rows, or those whose flag is not set, or whose word is not among n sorted keys
template <int NT> __device__ __forceinline__ void fill_zeros(const Fill& f, unsigned block, unsigned blocks) {
    fill_rows<NT>(f, block, blocks, [&](uint32_t, uint64_t row, bool in) __attribute__((always_inline)) {
        if (f.flags) return in && f.flags[row];
        if (!f.keys) return false;
        uint32_t lo = 0, hi = in ? f.n : 0;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (f.keys[mid] < row) lo = mid + 1; else hi = mid;
        }
        return in && lo < f.n && f.keys[lo] == row;
    });
}

// Digits of 64 places a wave at a time: lanes with the same digit find each other by comparing the digits' bits; a lane's rank is the number of lower lanes with its
// digit behind those that the wave has counted before.  count: the wave's own row of kDigits counters.
__device__ __forceinline__ uint32_t rank_in_wave(uint32_t digit, bool in, int bits, uint32_t* count) {
    uint64_t same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const uint64_t m = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? m : ~m;
    }
    const int lane = threadIdx.x & 63;
    const uint32_t lower = __popcll(same & ((1ull << lane) - 1));
    const uint32_t base = in ? count[digit] : 0;   // (one wave, one row: its LDS accesses are in order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && lower == 0) count[digit] = base + __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return base + lower;
}
// exclusive sums over the first kDigits threads of the workgroup
__device__ __forceinline__ uint32_t scan_digits(uint32_t v, uint32_t* lds) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t a = __shfl_up(s, o);
        if (lane >= o) s += a;
    }
    if (w < kDigits / kWave && lane == 63) lds[w] = s;
    __syncthreads();
    uint32_t before = 0;
    for (int i = 0; i < w && i < kDigits / kWave; ++i) before += lds[i];
    return before + s - v;
}

// Up to kSmall places: every place's rank is the number of (word, place) pairs below its own, counted over all pairs.  A workgroup has the pairs in its LDS, as one number each, and ranks
// kRanked places: lanes 16 apart and waves take different 64ths of the pairs.  4096 places are 17 M comparisons, two instructions each: 1 us of the whole chip, where a sort by one workgroup takes 15.
// The workgroups beyond fill.  (Ranking and filling workgroups by turns: 8192 places among 32000 words 32.9 us instead of 34.8, among 300 words 23.7 instead of 20.5.)
__global__ __launch_bounds__(kSortThreads) void rank_places_kernel(const void* __restrict__ tokens, bool index64, uint32_t n, uint32_t vocab, uint32_t* __restrict__ keys_out,
                                                                   uint32_t* __restrict__ places_out, uint32_t blocks, Fill fill) {
    constexpr uint32_t kParts = kSortThreads / kRanked;
    __shared__ __align__(16) uint32_t pairs[kSmall + 4 * kParts];
    __shared__ uint32_t ranks[kSortWaves][kRanked];
    if (blockIdx.x >= blocks) return fill_zeros<kSortThreads>(fill, blockIdx.x - blocks, gridDim.x - blocks);
    uint32_t part = (n + kParts - 1) / kParts;   // pairs of a 64th: whole reads of four, and 64ths that start in other banks
    part = (part + 3) / 4 * 4;
    if (part % 16 == 0) part += 4;
    for (uint32_t i = threadIdx.x; i < part * kParts; i += kSortThreads) pairs[i] = i < n ? key_of(tokens, index64, i, vocab) << kSmallBits | i : ~0u;
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * kRanked + lane % kRanked;
    const uint32_t own = pairs[i < n ? i : n - 1], *from = pairs + (threadIdx.x / kRanked) * part;
    uint32_t rank = 0;
#pragma unroll 4
    for (uint32_t j = 0; j < part; j += 4) {
        const uint4 four = *(const uint4*)(from + j);
        rank += (four.x < own) + (four.y < own) + (four.z < own) + (four.w < own);
    }
    rank += __shfl_xor(rank, 16);
    rank += __shfl_xor(rank, 32);
    if (lane < kRanked) ranks[w][lane] = rank;
    __syncthreads();
    if (threadIdx.x >= kRanked || i >= n) return;
    rank = 0;
#pragma unroll
    for (int v = 0; v < kSortWaves; ++v) rank += ranks[v][threadIdx.x];
    keys_out[rank] = own >> kSmallBits;
    places_out[rank] = i;
}

// One pass over more places (two launches of 5 and 8 us at 65536 places; counting the next digit in the same launch, with atomics, takes 29 us: half the words of a text share it): workgroup `tile` of `tiles`
// takes `span` of them.  FIRST: the first digit, straight from the tokens.
struct Pass {
    const void* tokens;
    const uint32_t *keys, *places;
    uint32_t *keys_out, *places_out, *counts;   // counts[tile][digit]
    uint8_t* flags;                             // of the words: cleared where the first digit is counted, set where its places are moved
    uint32_t n, span, tiles, vocab;
    int shift, bits, index64;
};
template <bool FIRST> __device__ __forceinline__ uint32_t key_at(const Pass& p, uint32_t i) { return FIRST ? key_of(p.tokens, p.index64, i, p.vocab) : p.keys[i]; }

template <bool FIRST> __global__ __launch_bounds__(kSortThreads) void count_digits_kernel(Pass p, Fill fill) {
    __shared__ uint32_t lds[kDigits];
    if (blockIdx.x >= p.tiles) {
        if (FIRST && p.flags)
            for (uint64_t i = (uint64_t)(blockIdx.x - p.tiles) * kSortThreads + threadIdx.x; i <= p.vocab; i += (uint64_t)(gridDim.x - p.tiles) * kSortThreads) p.flags[i] = 0;
        return fill_zeros<kSortThreads>(fill, blockIdx.x - p.tiles, gridDim.x - p.tiles);
    }
    const uint32_t mask = (1u << p.bits) - 1;
    if (threadIdx.x < kDigits) lds[threadIdx.x] = 0;
    __syncthreads();
    const uint64_t begin = (uint64_t)blockIdx.x * p.span, end = begin + p.span < p.n ? begin + p.span : p.n;
    for (uint64_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&lds[key_at<FIRST>(p, (uint32_t)i) >> p.shift & mask], 1u);   // (whole numbers: any order)
    __syncthreads();
    if (threadIdx.x < kDigits) p.counts[(size_t)blockIdx.x * kDigits + threadIdx.x] = lds[threadIdx.x];
}

template <bool FIRST> __global__ __launch_bounds__(kSortThreads) void move_places_kernel(Pass p, Fill fill) {
    __shared__ uint32_t counts[kSortWaves][kDigits], all[kSortThreads], before_me[kSortThreads], totals[kDigits / kWave];
    if (blockIdx.x >= p.tiles) return fill_zeros<kSortThreads>(fill, blockIdx.x - p.tiles, gridDim.x - p.tiles);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int wide = p.bits < 6 ? 6 : p.bits;   // (a digit has at most 16 threads in the sums of the counts)
    const uint32_t mask = (1u << p.bits) - 1, digits = 1u << wide;
    const uint64_t begin = (uint64_t)blockIdx.x * p.span, end = begin + p.span < p.n ? begin + p.span : p.n;
    uint32_t key[kTileRounds], rank[kTileRounds], place[kTileRounds];
    // (No branch around a load: lanes beyond the tile read its last place.  With `in ? ... : ...` around them the compiler has been seen to drop the copy of a place whose register the token had taken.)
    auto fetch = [&](uint64_t at) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kTileRounds; ++u) {
            const uint64_t i = at + (w * kTileRounds + u) * kWave + lane;
            place[u] = (uint32_t)(i < end ? i : end - 1);
            key[u] = key_at<FIRST>(p, place[u]);
        }
#pragma unroll
        for (int u = 0; u < kTileRounds; ++u) {
            if (!FIRST) place[u] = p.places[place[u]];
            if (at + (w * kTileRounds + u) * kWave + lane >= end) key[u] = ~0u;
        }
    };
    fetch(begin);
    // where this tile's places of each digit go: behind all smaller digits, and the same one in the tiles before.  The threads of a digit share the tiles, with eight loads on their way
    {
        const uint32_t parts = kSortThreads >> wide, each = (p.tiles + parts - 1) / parts, first = (threadIdx.x >> wide) * each, digit = threadIdx.x & (digits - 1);
        uint32_t total = 0, mine = 0;
        for (uint32_t t = 0; t < each; t += 8) {
            uint32_t c[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u] = p.counts[(size_t)(first + t + u < p.tiles ? first + t + u : p.tiles - 1) * kDigits + digit];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t tile = first + t + u, count = t + u < each && tile < p.tiles ? c[u] : 0;
                mine += tile < blockIdx.x ? count : 0;
                total += count;
            }
        }
        all[threadIdx.x] = total;
        before_me[threadIdx.x] = mine;
    }
    __syncthreads();
    uint32_t total = 0, next = 0;
    if (threadIdx.x < digits)
        for (uint32_t part = threadIdx.x; part < kSortThreads; part += digits) {
            total += all[part];
            next += before_me[part];
        }
    next += scan_digits(total, totals);   // (of the thread's digit)
    for (uint64_t at = begin; at < end; at += kSortThreads * kTileRounds) {
        if (at != begin) fetch(at);
        if (threadIdx.x <= mask)
#pragma unroll
            for (int v = 0; v < kSortWaves; ++v) counts[v][threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kTileRounds; ++u) rank[u] = rank_in_wave(key[u] >> p.shift & mask, key[u] != ~0u, p.bits, counts[w]);
        __syncthreads();
        if (threadIdx.x <= mask) {
            uint32_t c[kSortWaves];
#pragma unroll
            for (int v = 0; v < kSortWaves; ++v) c[v] = counts[v][threadIdx.x];
#pragma unroll
            for (int v = 0; v < kSortWaves; ++v) {
                counts[v][threadIdx.x] = next;
                next += c[v];
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kTileRounds; ++u)
            if (key[u] != ~0u) {
                if (FIRST && p.flags) p.flags[key[u]] = 1;
                const uint32_t to = counts[w][key[u] >> p.shift & mask] + rank[u];
                p.keys_out[to] = key[u];
                p.places_out[to] = place[u];
            }
        __syncthreads();
    }
}

// Groups of L lanes add up runs of `run` sorted places, kColumns columns a lane.  A word whose places all lie in the run is written to the table; the
// piece of a word that began in an earlier run goes to pieces[run][0], that of one that begins here and goes on to pieces[run][1].
// (65536 x 2048: runs of 64 leave every SIMD 8 waves with up to 16 rows each on their way; runs of 32 take as long and leave more pieces.)
struct Sum {
    const uint32_t *keys, *places;
    const void* dout;
    float *table, *pieces;
    uint32_t n, vocab, run;
    int width, accumulate;
    float scale;
    uint32_t column_blocks, blocks;   // of L * V columns; workgroups of the sums: further ones fill
};
// a word's sum to its row of the table, or, a piece of it, to `piece` (short code: it stands behind every place of a run)
template <bool ACCUMULATE, int V, bool NARROW> __device__ __forceinline__ void put_row(const Sum& q, const Columns<V, NARROW>& c, uint32_t word, float* piece, float (&s)[V]) {
    float* row = piece ? piece : q.table + (size_t)word * q.width;
    const float scale = piece ? 1.f : q.scale;
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] *= scale;
    if (ACCUMULATE && !piece) c.add(row, s);
    else c.store(row, s);
}

template <typename O, int L, bool NARROW, bool ACCUMULATE>
__global__ __launch_bounds__(kThreads) void sum_runs_kernel(Sum q, Fill fill) {
    constexpr int V = kColumns, kGroups = kThreads / L, kAhead = 8;
    if (blockIdx.x >= q.blocks) return fill_zeros<kThreads>(fill, blockIdx.x - q.blocks, gridDim.x - q.blocks);
    __shared__ uint32_t keys[kGroups][kMaxRun], places[kGroups][kMaxRun];   // of each group's run
    const int l = threadIdx.x % L, group = threadIdx.x / L;
    const uint32_t id = blockIdx.x * kGroups + group, r = id / q.column_blocks;   // (neighbours take a run's other columns: whole rows are read and written at about the same time)
    const uint64_t begin = (uint64_t)r * q.run;
    if (begin >= q.n) return;
    const uint32_t b = (uint32_t)begin, len = q.n - b < q.run ? q.n - b : q.run;
    for (uint32_t i = l; i < q.run; i += L) {
        const uint32_t at = b + (i < len ? i : len - 1);
        keys[group][i] = q.keys[at];
        places[group][i] = q.places[at];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a group lies in one wave)
    const uint32_t before = b ? q.keys[b - 1] : ~0u, after = b + len < q.n ? q.keys[b + len] : ~0u;
    const Columns<V, NARROW> col((id - r * q.column_blocks) * L + l, q.width);
    float* pieces = q.pieces + (size_t)r * 2 * q.width;
    uint32_t word = keys[group][0];
    float s[V] = {};
    Chunk<O, V> rows[2][kAhead];   // one set on its way while the other is added up
    auto fetch = [&](Chunk<O, V>(&row)[kAhead], uint32_t p) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) row[u] = col.load((const O*)q.dout + (size_t)places[group][p + u] * q.width);
    };
    auto add = [&](const Chunk<O, V>(&row)[kAhead], uint32_t p) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t key = keys[group][p + u];
            if (p + u < len) {
                if (key != word) {
                    put_row<ACCUMULATE>(q, col, word, word == before ? pieces : nullptr, s);   // (a word before another one is in the vocabulary)
                    word = key;
#pragma unroll
                    for (int i = 0; i < V; ++i) s[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] += row[u].get(i);
            }
        }
    };
    fetch(rows[0], 0);
    for (uint32_t p = 0; p < len; p += 2 * kAhead) {
        if (p + kAhead < len) fetch(rows[1], p + kAhead);
        add(rows[0], p);
        if (p + kAhead >= len) break;
        if (p + 2 * kAhead < len) fetch(rows[0], p + 2 * kAhead);
        add(rows[1], p + kAhead);
    }
    if (word == q.vocab) return;
    put_row<ACCUMULATE>(q, col, word, word == before ? pieces : word == after ? pieces + q.width : nullptr, s);
}

// Where a word begins in a run and goes on beyond it, its pieces are added up in order and its row is written.  Most such words go on through one or two runs: a group of L lanes per run (and L * kColumns
// columns) adds them up, behind the first `longs` workgroups.  These have one window of kManyRuns runs each, in which at most one word can begin that goes on through kManyRuns or more: the whole
// workgroup looks for its end and adds it up, its groups every kGroups-th piece.  (A workgroup for every run instead: 18750 runs of 64 columns take 2 us more,
// 31250 of 64 columns, with words of thousands of runs, 6 us.)
constexpr int kManyRuns = 8;
template <int L, bool NARROW>
__global__ __launch_bounds__(kThreads) void join_pieces_kernel(Sum q, uint32_t runs, uint32_t longs) {
    constexpr int V = kColumns, kGroups = kThreads / L;
    __shared__ float lds[kGroups][L][V];
    const int lane = threadIdx.x & 63, l = threadIdx.x % L;
    const uint32_t group = threadIdx.x / L;
    const bool is_long = blockIdx.x < longs;
    const Columns<V, NARROW> col(blockIdx.y * L + l, q.width);
    const size_t step = 2 * (size_t)q.width;
    // s += pieces k, k + by, ... up to `last` of those at `from`, AHEAD of them on their way
    auto add = [&](auto ahead, float(&s)[V], const float* from, uint32_t k, uint32_t by, uint32_t last) __attribute__((always_inline)) {
        constexpr int kAhead = decltype(ahead)::value;
        for (; k <= last; k += kAhead * by) {
            Chunk<float, V> c[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) c[u] = col.load(from + (k + u * by <= last ? k + u * by : last) * step);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (k + u * by <= last)
#pragma unroll
                    for (int i = 0; i < V; ++i) s[i] += c[u].get(i);
        }
    };
    auto begin = [&](float(&s)[V], const float* from) __attribute__((always_inline)) {   // the piece in the run itself
        const Chunk<float, V> c = col.load(from + q.width);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = c.get(i);
    };
    auto put = [&](uint32_t word, float(&s)[V]) __attribute__((always_inline)) {
        if (q.accumulate) put_row<true>(q, col, word, nullptr, s);
        else put_row<false>(q, col, word, nullptr, s);
    };
    // the word that run r ends with, if it begins there and goes on, or else vocab
    auto word_from = [&](uint32_t r) __attribute__((always_inline)) {
        if (r + 1 >= runs) return q.vocab;
        const uint32_t b = r * q.run, e = b + q.run, before = q.keys[b ? b - 1 : 0], word = q.keys[e - 1];
        return q.keys[e] == word && !(b && before == word) ? word : q.vocab;
    };
    auto begins_with = [&](uint32_t r, uint32_t word) __attribute__((always_inline)) { return r < runs && q.keys[r < runs ? (size_t)r * q.run : 0] == word; };
    if (!is_long) {
        const uint32_t r = (blockIdx.x - longs) * kGroups + group, word = word_from(r);
        // runs that it goes on through: those that begin with it, of the next kManyRuns
        const uint64_t m = __ballot(word != q.vocab && l < kManyRuns && begins_with(r + 1 + l, word)) >> (lane - l);
        const int more = __builtin_ctzll(~(m & ((1ull << kManyRuns) - 1)));
        if (more == 0 || more == kManyRuns) return;
        const float* from = q.pieces + (size_t)r * step;
        float s[V];
        begin(s, from);
        add(Int<4>{}, s, from, 1, 1, more);
        put(word, s);
        return;
    }
    const uint32_t first = blockIdx.x * kManyRuns + lane % kManyRuns, mine = word_from(first);
    const uint64_t there = __ballot(mine != q.vocab && begins_with(first + kManyRuns, mine));
    if (!there) return;
    const uint32_t r = blockIdx.x * kManyRuns + __builtin_ctzll(there), word = q.keys[(size_t)(r + 1) * q.run];
    uint32_t lo = r + 1 + kManyRuns, hi = runs;   // run lo - 1 begins with the word, run hi does not, or is none: 64 between them are looked at at a time
    while (lo < hi) {
        const uint32_t part = (hi - lo + kWave - 1) / kWave;
        const uint32_t n = __popcll(__ballot(lo + lane * part < hi && begins_with(lo + lane * part, word))), to = lo + n * part;
        hi = n == 0 ? lo : to < hi ? to : hi;
        lo = n == 0 ? lo : lo + (n - 1) * part + 1;
    }
    const uint32_t more = lo - 1 - r;
    const float* from = q.pieces + (size_t)r * step;
    float s[V] = {};
    if (group == 0) begin(s, from);
    add(Int<8>{}, s, from, 1 + group, kGroups, more);
#pragma unroll
    for (int i = 0; i < V; ++i) lds[group][l][i] = s[i];
    __syncthreads();
    if (group) return;
    const uint32_t groups = more + 1 < (uint32_t)kGroups ? more + 1 : kGroups;   // (that have added anything)
    for (uint32_t v = 1; v < groups; ++v)
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] += lds[v][l][i];
    put(word, s);
}

// Up to kFewPlaces places, one launch: a workgroup per place (and L * kColumns columns) looks for the places of its word and, where none comes before its own, adds them up: each group of L lanes a part
// of them, in order, and the parts in order.  The workgroups beyond fill, with the words in their registers.  Every workgroup reads all tokens, so there are up to kFewBlocks of them (1024 places of 4096
// columns 29 us, by sorting 13.8); and all places may have one word, so a group gets up to kFewRows of them (with the loads of 16 or 32 of its rows on their way instead of 8 this is no faster: the wave's own
// instructions bound it).  Half of the places one word's, the others among 300 words: 256 of 768 columns 5.8 us and,
// by sorting, 11.3; 512 8.5 and 11.3 (all one word's: 13.7 and 11.3); 1024 13.6 and 11.4 (23.8 and 12.5); 1024 of 64 columns 6.4 and 11.3 (9.2 and 11.1).
constexpr uint32_t kFewPlaces = 1024, kFewBlocks = 4096, kFewRows = 128;
template <typename O, int L, bool NARROW, bool ACCUMULATE>
__global__ __launch_bounds__(kThreads) void few_places_kernel(Sum q, const void* tokens, bool index64, Fill fill) {
    constexpr int V = kColumns, kGroups = kThreads / L, kAhead = 8, kWaves = kThreads / kWave, kParts = kFewPlaces / kWave;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (blockIdx.x >= q.blocks) {
        __shared__ uint32_t words[kWaves][2];
        uint32_t keys[kParts];   // (no row's number: none)
#pragma unroll
        for (int u = 0; u < kParts; ++u) {
            const uint32_t i = u * kWave + lane, key = i < q.n ? key_of(tokens, index64, i, q.vocab) : q.vocab;
            keys[u] = key < q.vocab ? key : ~0u;
        }
        return fill_rows<kThreads>(fill, blockIdx.x - q.blocks, gridDim.x - q.blocks, [&](uint32_t first, uint64_t, bool) __attribute__((always_inline)) {
            bool any = false;
#pragma unroll
            for (int u = 0; u < kParts; ++u) any |= keys[u] - first < fill.each;
            if (!__ballot(any)) return false;
            if (lane < 2) words[w][lane] = 0;   // (one wave: its LDS accesses are in order)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int u = 0; u < kParts; ++u)
                if (keys[u] - first < fill.each) atomicOr(&words[w][(keys[u] - first) / 32], 1u << (keys[u] - first) % 32);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const bool there = words[w][lane / 32] >> lane % 32 & 1;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            return there;
        });
    }
    __shared__ uint64_t masks[kParts];
    __shared__ uint32_t places[kFewPlaces];
    __shared__ float lds[kGroups][L][V];
    const uint32_t own = blockIdx.x / q.column_blocks, word = key_of(tokens, index64, own, q.vocab);
    if (word == q.vocab) return;
    uint64_t mask[kParts / kWaves];   // places of the word, 64 at a time; the wave's
#pragma unroll
    for (int u = 0; u < kParts / kWaves; ++u) {
        const uint32_t i = u * kThreads + threadIdx.x;
        mask[u] = __ballot(key_of(tokens, index64, i < q.n ? i : q.n - 1, q.vocab) == word && i < q.n);
        if (lane == 0) masks[u * kWaves + w] = mask[u];
    }
    __syncthreads();
    uint32_t total = 0, earlier = 0;   // places of the word: all, before the workgroup's own
#pragma unroll
    for (int v = 0; v < kParts; ++v) {
        const uint64_t m = masks[v];
        if (v == (int)(own / kWave)) earlier = total + __popcll(m & ((1ull << own % kWave) - 1));
        if (v % kWaves == w && mask[v / kWaves] >> lane & 1) places[total + __popcll(m & ((1ull << lane) - 1))] = v * kWave + lane;
        total += __popcll(m);
    }
    if (earlier) return;
    __syncthreads();
    const int l = threadIdx.x % L;
    const uint32_t group = threadIdx.x / L, part = (total + kGroups - 1) / kGroups, end = (group + 1) * part < total ? (group + 1) * part : total;
    const Columns<V, NARROW> col((blockIdx.x - own * q.column_blocks) * L + l, q.width);
    float s[V] = {};
    for (uint32_t k = group * part; k < end; k += kAhead) {
        Chunk<O, V> rows[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) rows[u] = col.load((const O*)q.dout + (size_t)places[k + u < end ? k + u : end - 1] * q.width);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (k + u < end)
#pragma unroll
                for (int c = 0; c < V; ++c) s[c] += rows[u].get(c);
    }
    if (total > 1) {
#pragma unroll
        for (int c = 0; c < V; ++c) lds[group][l][c] = s[c];
        __syncthreads();
    }
    if (group) return;
    for (uint32_t v = 1; v * part < total; ++v)
#pragma unroll
        for (int c = 0; c < V; ++c) s[c] += lds[v][l][c];
    put_row<ACCUMULATE>(q, col, word, nullptr, s);
}

int check_desc(const flashrnn_embedding_desc_t* d, bool gradient) {
    if (!d) return FLASHRNN_ERR_NULL;
    if (d->tokens < 0 || d->vocab <= 0 || d->width <= 0) return FLASHRNN_ERR_SHAPE;
    if (!is_io_type(d->table_dtype) || !is_io_type(d->io_dtype) || !is_index_type(d->index_dtype)) return FLASHRNN_ERR_SHAPE;
    // every offset below 2^62 bytes; the gradient's workgroups (one per run of places, and so on) below 2^32 threads, 2^16 in the other direction
    if ((double)d->tokens * d->width > 1e18 || d->width > (1 << 20) || (gradient && d->tokens >= (1LL << 29))) return FLASHRNN_ERR_UNSUPPORTED;
    return FLASHRNN_OK;
}

// lanes per row: the number that leaves the fewest of them without columns, the larger one of equals.  (A width with a small remainder gets few lanes and many blocks of columns, as 1100 does with 8 and 35: fewer
// of its places go into one launch, up to 117 where 1024 columns allow 512, and 16384 of them among 32000 words take 57.7 us, of 1152 columns 52.8.)
int lanes_for(int chunks) {
    int best = 64;
    for (int L = 32; L >= 8; L /= 2)
        if ((chunks + L - 1) / L * L < (chunks + best - 1) / best * best) best = L;
    return best;
}

// How the gradient is laid out: the sort's passes and tiles, the runs, the workspace.
struct Plan {
    int passes, bits;
    uint32_t tiles, span;   // tiles = 0: sorted by counting
    int L, column_blocks;
    uint32_t run, runs;
    size_t keys[2], places[2], counts, flags, pieces, total;
};
Plan plan_of(const flashrnn_embedding_desc_t* d) {
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    Plan p;
    const size_t n = (size_t)d->tokens;
    int bits = 1;
    while ((uint64_t)d->vocab >> bits) ++bits;   // keys go up to vocab itself
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = p.span = 0;
    if (n > kSmall || (uint32_t)d->vocab >> (32 - kSmallBits)) {   // (word and place have to fit into 32 bits, with one number left above them all)
        const size_t step = kSortThreads * kTileRounds, steps = (n + step - 1) / step, each = (steps + kMaxTiles - 1) / kMaxTiles;
        p.span = (uint32_t)(each * step);
        p.tiles = (uint32_t)((n + p.span - 1) / p.span);
    }
    const int chunks = (d->width + kColumns - 1) / kColumns;
    p.L = lanes_for(chunks);
    p.column_blocks = (chunks + p.L - 1) / p.L;
    // places per run: enough runs for 2048 waves, as long as that leaves them kMinRun places or more
    const size_t waves = n * p.column_blocks * p.L / kWave;
    p.run = kMaxRun;
    while (p.run > kMinRun && waves / p.run < 2048) p.run /= 2;
    p.runs = (uint32_t)((n + p.run - 1) / p.run);
    size_t at = 0;
    const size_t list = up(n * 4);
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = at; at += list;
        p.places[i] = at; at += list;
    }
    p.counts = at; at += up((size_t)p.tiles * kDigits * 4);
    p.flags = at; at += p.tiles ? up((size_t)d->vocab + 1) : 0;
    p.pieces = at; at += up((size_t)p.runs * 2 * d->width * 4);
    p.total = at + 256;
    return p;
}

}  // namespace

extern "C" {

size_t flashrnn_embedding_workspace_bytes(const flashrnn_embedding_desc_t* d) { return check_desc(d, true) == FLASHRNN_OK ? plan_of(d).total : 0; }

int flashrnn_embedding_fwd(const flashrnn_embedding_desc_t* d, const void* table, const void* tokens, void* out, void* hip_stream) {
    const int rc = check_desc(d, false);
    if (rc != FLASHRNN_OK) return rc;
    if (d->tokens == 0) return FLASHRNN_OK;
    if (!table || !tokens || !out) return FLASHRNN_ERR_NULL;
    if (!aligned_to(table, type_size(d->table_dtype)) || !aligned_to(out, type_size(d->io_dtype)) || !aligned_to(tokens, type_size(d->index_dtype))) return FLASHRNN_ERR_UNSUPPORTED;
    return with_io_type(d->table_dtype, [&](auto* et) {
        return with_io_type(d->io_dtype, [&](auto* ot) {
            using E = std::remove_pointer_t<decltype(et)>;
            using O = std::remove_pointer_t<decltype(ot)>;
            constexpr int V = sizeof(E) == 2 && sizeof(O) == 2 ? 8 : 4;
            const int chunks = (d->width + V - 1) / V, L = lanes_for(chunks);
            const uint64_t n = (uint64_t)d->tokens;
            const uint32_t column_blocks = (uint32_t)((chunks + L - 1) / L);
            const Lookup q{table, tokens, out, n, (uint32_t)d->vocab, column_blocks, d->width, d->index_dtype == FLASHRNN_I64, n * d->width * sizeof(O) > kStreamBytes, d->scale};
            const bool many = n * column_blocks * L / kWave >= kManyWaves;
            auto launch = [&](auto lanes, auto narrow) {
                constexpr int kLanes = decltype(lanes)::value;
                constexpr bool kNarrow = decltype(narrow)::value;
                const uint64_t groups = (n + (many ? kRows : 1) - 1) / (many ? kRows : 1) * column_blocks;
                const dim3 grid(row_blocks((groups + kThreads / kLanes - 1) / (kThreads / kLanes)));
                if (many) hipLaunchKernelGGL((embedding_fwd_kernel<E, O, kLanes, kRows, kNarrow>), grid, dim3(kThreads), 0, (hipStream_t)hip_stream, q);
                else hipLaunchKernelGGL((embedding_fwd_kernel<E, O, kLanes, 1, kNarrow>), grid, dim3(kThreads), 0, (hipStream_t)hip_stream, q);
            };
            if (d->width < V) launch(Int<8>{}, Int<1>{});
            else if (L == 64) launch(Int<64>{}, Int<0>{});
            else if (L == 32) launch(Int<32>{}, Int<0>{});
            else if (L == 16) launch(Int<16>{}, Int<0>{});
            else launch(Int<8>{}, Int<0>{});
            return launch_status();
        });
    });
}

int flashrnn_embedding_bwd(const flashrnn_embedding_desc_t* d, const void* tokens, const void* dout, void* dtable, int accumulate, void* workspace, void* hip_stream) {
    const int rc = check_desc(d, true);
    if (rc != FLASHRNN_OK) return rc;
    const size_t n = (size_t)d->tokens;
    if (!dtable || (n && (!tokens || !dout))) return FLASHRNN_ERR_NULL;
    if (!workspace || !aligned_to(workspace, 256)) return FLASHRNN_ERR_WORKSPACE;
    if (!aligned_to(dout, type_size(d->io_dtype)) || !aligned_to(tokens, type_size(d->index_dtype)) || !aligned_to(dtable, 4)) return FLASHRNN_ERR_UNSUPPORTED;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const Plan p = plan_of(d);
    if ((double)p.runs * p.column_blocks * p.L >= 4e9) return FLASHRNN_ERR_UNSUPPORTED;   // (more than any memory holds)
    char* ws = (char*)workspace;
    const size_t row_bytes = (size_t)d->width * 4;
    Fill fill{(float*)dtable, nullptr, nullptr, 0, 0, (uint32_t)(row_bytes >= kFillBytes ? 1 : row_bytes * kWave <= kFillBytes ? kWave : kFillBytes / row_bytes), (uint32_t)n, d->width};
    auto fill_to = [&](uint32_t end, int waves) {   // the rows behind those filled so far; the workgroups for them
        fill.begin = fill.end;
        fill.end = accumulate ? 0 : end;
        const size_t parts = ((size_t)fill.end - fill.begin + fill.each - 1) / fill.each, blocks = (parts + waves - 1) / waves;
        return (unsigned)(blocks < kFillWaves / waves ? blocks : kFillWaves / waves);
    };
    const uint32_t vocab = (uint32_t)d->vocab;
    auto by_lanes = [&](auto&& launch) {
        if (d->width < kColumns) launch(Int<8>{}, Int<1>{});
        else if (p.L == 64) launch(Int<64>{}, Int<0>{});
        else if (p.L == 32) launch(Int<32>{}, Int<0>{});
        else if (p.L == 16) launch(Int<16>{}, Int<0>{});
        else launch(Int<8>{}, Int<0>{});
        return launch_status();
    };
    if (n <= kFewPlaces && n * p.column_blocks <= kFewBlocks && n * p.L <= kFewRows * kThreads) {
        const unsigned fills = fill_to(vocab, kThreads / kWave), blocks = (unsigned)n * p.column_blocks;
        if (blocks + fills == 0) return FLASHRNN_OK;
        const Sum q{nullptr, nullptr, dout, (float*)dtable, nullptr, (uint32_t)n, vocab, 0, d->width, accumulate, d->scale, (uint32_t)p.column_blocks, blocks};
        return with_io_type(d->io_dtype, [&](auto* ot) {
            using O = std::remove_pointer_t<decltype(ot)>;
            return by_lanes([&](auto lanes, auto narrow) {
                auto kernel = accumulate ? few_places_kernel<O, decltype(lanes)::value, decltype(narrow)::value, true> : few_places_kernel<O, decltype(lanes)::value, decltype(narrow)::value, false>;
                hipLaunchKernelGGL(kernel, dim3(blocks + fills), dim3(kThreads), 0, stream, q, tokens, d->index_dtype == FLASHRNN_I64, fill);
            });
        });
    }
    auto fill_beside = [&] { return kFillBesideSort / row_bytes < vocab - fill.end ? fill.end + (uint32_t)(kFillBesideSort / row_bytes) : vocab; };
    uint32_t *keys = (uint32_t*)(ws + p.keys[0]), *places = (uint32_t*)(ws + p.places[0]);
    if (p.tiles == 0) {
        const uint32_t part = (uint32_t)(kFillBesideSums / row_bytes);
        const unsigned fills = fill_to(vocab <= part ? vocab : vocab <= 2 * part ? part : vocab - part, kSortWaves), blocks = (unsigned)((n + kRanked - 1) / kRanked);
        hipLaunchKernelGGL(rank_places_kernel, dim3(blocks + fills), dim3(kSortThreads), 0, stream, tokens, d->index_dtype == FLASHRNN_I64, (uint32_t)n, vocab, keys, places, blocks, fill);
        if (const int e = launch_status()) return e;
        fill.keys = keys;
    } else {
        uint8_t* flags = accumulate ? nullptr : (uint8_t*)(ws + p.flags);
        Pass q{tokens, nullptr, nullptr, nullptr, nullptr, (uint32_t*)(ws + p.counts), flags, (uint32_t)n, p.span, p.tiles, vocab, 0, p.bits, d->index_dtype == FLASHRNN_I64};
        for (int pass = 0; pass < p.passes; ++pass) {
            q.shift = pass * p.bits;
            q.keys_out = keys = (uint32_t*)(ws + p.keys[pass & 1]);
            q.places_out = places = (uint32_t*)(ws + p.places[pass & 1]);
            for (int step = 0; step < 2; ++step) {
                unsigned more = 0;   // workgroups beside the sort
                if (pass) more = fill_to(fill_beside(), kSortWaves);
                else if (step == 0 && flags) more = vocab / kFlagsPerBlock < kFlagBlocks ? 1 + vocab / kFlagsPerBlock : kFlagBlocks;
                const dim3 grid(p.tiles + more);
                if (step == 0) hipLaunchKernelGGL((pass ? count_digits_kernel<false> : count_digits_kernel<true>), grid, dim3(kSortThreads), 0, stream, q, fill);
                else hipLaunchKernelGGL((pass ? move_places_kernel<false> : move_places_kernel<true>), grid, dim3(kSortThreads), 0, stream, q, fill);
                if (const int e = launch_status()) return e;
                fill.flags = flags;
            }
            q.keys = keys;
            q.places = places;
        }
    }
    const unsigned fill_blocks = fill_to(vocab, kThreads / kWave);   // (with few places: none are left)
    const uint32_t sum_blocks = (uint32_t)(((size_t)p.runs * p.column_blocks + kThreads / p.L - 1) / (kThreads / p.L));
    const Sum q{keys, places, dout, (float*)dtable, (float*)(ws + p.pieces), (uint32_t)n, vocab, p.run, d->width, accumulate, d->scale, (uint32_t)p.column_blocks, sum_blocks};
    const int e = with_io_type(d->io_dtype, [&](auto* ot) {
        using O = std::remove_pointer_t<decltype(ot)>;
        const dim3 grid(sum_blocks + fill_blocks);
        return by_lanes([&](auto lanes, auto narrow) {
            if (accumulate) hipLaunchKernelGGL((sum_runs_kernel<O, decltype(lanes)::value, decltype(narrow)::value, true>), grid, dim3(kThreads), 0, stream, q, fill);
            else hipLaunchKernelGGL((sum_runs_kernel<O, decltype(lanes)::value, decltype(narrow)::value, false>), grid, dim3(kThreads), 0, stream, q, fill);
        });
    });
    if (e != FLASHRNN_OK) return e;
    return by_lanes([&](auto lanes, auto narrow) {
        constexpr unsigned kGroups = kThreads / decltype(lanes)::value;
        const unsigned longs = (p.runs + kManyRuns - 1) / kManyRuns;
        hipLaunchKernelGGL((join_pieces_kernel<decltype(lanes)::value, decltype(narrow)::value>), dim3(longs + (p.runs + kGroups - 1) / kGroups, p.column_blocks), dim3(kThreads), 0, stream, q, p.runs, longs);
    });
}

}  // extern "C"
