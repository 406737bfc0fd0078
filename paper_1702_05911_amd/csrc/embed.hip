// Rows of an embedding table for tokens, scaled, and the table's gradient.
//
// Lookup: out[t] = scale * table[tokens[t]].  Bound by memory: a row is read and written once.  A group of lanes (as many as the
// row has pieces of 16 bytes, up to a wavefront) has a row or a section of one, up to four pieces a lane, all loaded before the first is
// stored; 2,048 workgroups walk the tokens, the next one's number read ahead.  100,003 rows of 1,024, bf16 to floats: 78 us, 5.9 TB/s
// of what has to move (a large copy 5.1, a fill 6.9: most of it is writing).  7 rows: 2.3 us, less than a launch.
//
// Gradient: out[v] = scale * sum of grad[t] over the places of v.  Additions by atomics would give other bits on every call and
// queue up at the tokens that are in every sentence, so the places are sorted by token first: digits of up to ten bits from
// the lowest on, every pass stable, so that a token's places ascend.  The sort fills few compute units and waits for memory; the others
// clear the result meanwhile.  Then the sorted places are walked in chunks of equal length, one a group of lanes, whatever
// tokens they belong to: rows are read eight at a time, and where the token changes the sum so far goes out.  A token that lies in one
// chunk is finished there; of the others the chunks' parts go to the workspace, and join_kernel adds them in order.  Up to kRankPlaces are
// put in order by one launch, and a few places need none (few_places).
// Bound by memory: n rows read, V written; the sort moves 16 bytes a place and pass.  131,071 places of 1,024 bf16 values, 65,536 rows of
// floats: 150 us, of it two passes of the sort, with the zeros, 54, the sums 84, the joining 11; the bytes alone, at a copy's rate,
// 103.  Sums in fp32, rounded once.
#include <algorithm>

#include "encoder.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int64_t kMaxEmbedD = 1 << 20;    // (sections of a row are the grid's second dimension: 2^16 - 1 at most)
constexpr int64_t kMaxPlaces = 0x7fffffff; // places are 32-bit numbers
constexpr int64_t kMaxRows = 1 << 28;      // of a gradient (32 a workgroup of 256, of 2^32 threads in all)
constexpr int kEmbedBlocks = 2048;         // workgroups of a lookup: what fits the compute units, each walks the tokens

struct EmbedArgs {
    const void* table;
    const void* tokens;
    void* out;
    int64_t V, D, table_stride, n, out_stride;
    float scale;
    int log_lanes;                         // lanes of a row's section, log2
    int wide_tokens;
    int stream;                            // store past the caches
};

__device__ __forceinline__ int64_t token_at(const void* tokens, int wide, int64_t i) {
    return wide ? static_cast<const int64_t*>(tokens)[i] : (int64_t) static_cast<const int32_t*>(tokens)[i];
}

// NP: pieces of a row that a lane has
template <typename TX, typename TY, int NP>
__global__ __launch_bounds__(kEmbedThreads) void embed_kernel(EmbedArgs g) {
    constexpr int E = sizeof(TX) == 2 && sizeof(TY) == 2 ? 8 : 4;           // elements of a piece
    const int lanes = 1 << g.log_lanes, l = threadIdx.x & (lanes - 1);
    const int64_t per_block = kEmbedThreads >> g.log_lanes;
    const int64_t col = ((int64_t)blockIdx.y * NP * lanes + l) * E, step = (int64_t)gridDim.x * per_block;
    int64_t t = (int64_t)blockIdx.x * per_block + (threadIdx.x >> g.log_lanes);
    int64_t next = t < g.n ? token_at(g.tokens, g.wide_tokens, t) : 0;
    for (; t < g.n; t += step) {
        const int64_t v = next;
        const bool have = v >= 0 && v < g.V;
        const TX* src = static_cast<const TX*>(g.table) + (have ? v : 0) * g.table_stride;
        TY* dst = static_cast<TY*>(g.out) + t * g.out_stride;
        next = token_at(g.tokens, g.wide_tokens, min(t + step, g.n - 1));
        if (g.D < E) {                                                         // a row of fewer values than a piece
            for (int j = 0; j < (int)g.D; ++j)
                if (l == 0) dst[j] = from_float<TY>(have ? to_float(src[j]) * g.scale : 0.0f);
            continue;
        }
        typename Piece_<TX, E>::type r[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) r[p] = WholePiece<E>(col + (int64_t)p * lanes * E, g.D).template load<TX>(src);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int64_t c = col + (int64_t)p * lanes * E;
            typename Floats<E>::type f = __builtin_convertvector(r[p], typename Floats<E>::type) * g.scale;
            if (!have) f = 0.0f;                                               // (row 0 stood in)
            if (c < g.D) WholePiece<E>(c, g.D).template store<TY>(dst, f, g.stream);
        }
    }
}

// ---- gradient: places by token ---------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortBits = 10, kSortBins = 1 << kSortBits;
// Places of a tile of the sort (2,048: a pass over 131,071 places takes 27 us, 4,096: 30, half the tiles but twice the rounds of each), more
// where there would be more tiles than kSortTiles: a tile adds up the counts of all of them itself.
constexpr int64_t kSortTile = 2048, kSortTiles = 128;

struct SortArgs {
    const void* tokens;
    int wide_tokens;
    uint32_t n, V, tile;                   // tile: places of a workgroup, a multiple of kSortThreads
    uint32_t* key[2];                      // sorted tokens (V for those outside 0 .. V-1) and their places, to and fro
    uint32_t* place[2];
    uint32_t* counts;                      // tiles x kSortBins
    int passes, bits;                      // bits of a digit
};

// Zeros for the whole gradient, written beside the sort, whose workgroups leave most of the compute units idle; what has a sum is
// written again later.  In units of a row, or where rows follow each other of kClearUnit bytes.
constexpr int64_t kClearUnit = 4096;
constexpr int64_t kClearBlocks = 448;      // two workgroups on most compute units
struct ClearArgs {
    unsigned char* out;
    int64_t unit, step, total;             // bytes of a unit, from unit to unit, of all units (the last may be shorter)
    int64_t first, last;                   // units of this launch
    int stream;
};

// by workgroup `block` of `blocks`, a unit a wavefront
__device__ __forceinline__ void clear_units(const ClearArgs& c, uint32_t block, uint32_t blocks) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
    const int lane = threadIdx.x & (kWave - 1), waves = blockDim.x / kWave;
    for (int64_t u = c.first + (int64_t)block * waves + threadIdx.x / kWave; u < c.last; u += (int64_t)blocks * waves) {
        unsigned char* p = c.out + u * c.step;
        const int64_t len = min(c.unit, c.total - u * c.unit);
        for (int64_t at = lane * 16; at < len; at += kWave * 16) {
            if (at + 16 <= len) store_vector(reinterpret_cast<u32x4*>(p + at), u32x4{0u, 0u, 0u, 0u}, c.stream);
            else
                for (int64_t b = at; b < len; b += 2) *reinterpret_cast<uint16_t*>(p + b) = 0;
        }
    }
}

__device__ __forceinline__ uint32_t key_of(const SortArgs& g, int pass, uint32_t i) {
    if (pass) return g.key[(pass - 1) & 1][i];
    const int64_t v = token_at(g.tokens, g.wide_tokens, i);
    return v >= 0 && v < (int64_t)g.V ? (uint32_t)v : g.V;
}

constexpr int kSortE = 4;                  // keys of a thread on their way at a time

// how often every digit occurs in the tile
__device__ void count_digits(const SortArgs& g, int pass, uint32_t first, uint32_t* hist) {
    const int shift = pass * g.bits;
    const uint32_t mask = (1u << g.bits) - 1u;
    for (uint32_t b = threadIdx.x; b < kSortBins; b += kSortThreads) hist[b] = 0u;
    __syncthreads();
    for (uint32_t i = first + threadIdx.x; i < first + g.tile; i += kSortThreads * kSortE) {
        uint32_t key[kSortE];
#pragma unroll
        for (uint32_t u = 0; u < kSortE; ++u) key[u] = key_of(g, pass, min(i + u * kSortThreads, g.n - 1));
#pragma unroll
        for (uint32_t u = 0; u < kSortE; ++u)
            if (i + u * kSortThreads < min(g.n, first + g.tile)) atomicAdd(&hist[(key[u] >> shift) & mask], 1u);
    }
    __syncthreads();
}

// Places of one tile, stable: every wavefront has a consecutive part of the tile and counters of its own, which start where its
// digits' places start.  before / all: the digit's places in the tiles before this one, and in all of them (threadIdx.x is the digit).
__device__ void place_digits(const SortArgs& g, int pass, uint32_t first, uint32_t before, uint32_t all, uint32_t (*next)[kSortBins], uint32_t* part) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int shift = pass * g.bits;
    const uint32_t mask = (1u << g.bits) - 1u, len = g.tile / kSortWaves;
    const uint32_t bins = 1u << g.bits;
    uint32_t* out_key = g.key[pass & 1];
    uint32_t* out_place = g.place[pass & 1];
    if ((uint32_t)tid < bins)
        for (int w = 0; w < kSortWaves; ++w) next[w][tid] = 0u;
    __syncthreads();
    const uint32_t lo = first + wave * len, end = min(g.n, lo + len);     // (lo may lie past the last place)
    auto look = [&](uint32_t i, uint32_t (&key)[kSortE], uint32_t (&place)[kSortE]) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t u = 0; u < kSortE; ++u) {
            const uint32_t from = min(i + u * kWave, g.n - 1);
            key[u] = key_of(g, pass, from);
            place[u] = pass ? g.place[(pass - 1) & 1][from] : from;
        }
    };
    uint32_t first_key[kSortE], first_place[kSortE];                      // of the first round, which is mostly the only one
    look(lo + lane, first_key, first_place);
    for (uint32_t i = lo + lane; i - lane < end; i += kWave * kSortE) {
        uint32_t key[kSortE], place[kSortE];
        if (i == lo + lane) {
#pragma unroll
            for (int u = 0; u < kSortE; ++u) key[u] = first_key[u];
        } else look(i, key, place);
#pragma unroll
        for (uint32_t u = 0; u < kSortE; ++u)
            if (i + u * kWave < end) atomicAdd(&next[wave][(key[u] >> shift) & mask], 1u);
    }
    uint32_t total;
    uint32_t at = block_exclusive_sum(all, part, total) + before;         // (a barrier inside)
    __syncthreads();
    if ((uint32_t)tid < bins) {
        uint32_t c[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) c[w] = next[w][tid];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            next[w][tid] = at;
            at += c[w];
        }
    }
    __syncthreads();
    for (uint32_t i = lo + lane; i - lane < end; i += kWave * kSortE) {
        uint32_t key[kSortE], place[kSortE];
        if (i == lo + lane) {
#pragma unroll
            for (int u = 0; u < kSortE; ++u) {
                key[u] = first_key[u];
                place[u] = first_place[u];
            }
        } else look(i, key, place);
#pragma unroll
        for (uint32_t u = 0; u < kSortE; ++u) {
            if (i - lane + u * kWave >= end) break;                       // (the same for the wavefront)
            const bool have = i + u * kWave < end;
            const uint32_t digit = (key[u] >> shift) & mask;
            unsigned long long same = __ballot(have);
            for (int b = 0; b < g.bits; ++b) {
                const unsigned long long one = __ballot((digit >> b) & 1u);
                same &= (digit >> b) & 1u ? one : ~one;
            }
            const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
            const uint32_t from = have ? next[wave][digit] : 0u;
            wave_lds_order();
            if (have) {
                if (rank == 0) next[wave][digit] = from + (uint32_t)__popcll(same);
                out_key[from + rank] = key[u];
                out_place[from + rank] = place[u];
            }
            wave_lds_order();
        }
    }
}

__global__ __launch_bounds__(kSortThreads) void token_counts_kernel(SortArgs g, int pass, uint32_t tiles, ClearArgs clear) {
    __shared__ uint32_t hist[kSortBins];
    if (blockIdx.x >= tiles) {
        clear_units(clear, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    count_digits(g, pass, blockIdx.x * g.tile, hist);
    for (uint32_t b = threadIdx.x; b < kSortBins; b += kSortThreads) g.counts[(size_t)blockIdx.x * kSortBins + b] = hist[b];
}

__global__ __launch_bounds__(kSortThreads) void token_places_kernel(SortArgs g, int pass, uint32_t tiles, ClearArgs clear) {
    __shared__ uint32_t next[kSortWaves][kSortBins];
    __shared__ uint32_t part[kSortWaves];
    if (blockIdx.x >= tiles) {
        clear_units(clear, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    uint32_t before = 0, all = 0;
    constexpr uint32_t kAtOnce = 32;                          // tiles' counts on their way
    for (uint32_t t = 0; t < tiles; t += kAtOnce) {
        uint32_t c[kAtOnce];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) c[u] = g.counts[(size_t)min(t + u, tiles - 1) * kSortBins + threadIdx.x];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            before += t + u < blockIdx.x ? c[u] : 0u;
            all += t + u < tiles ? c[u] : 0u;
        }
    }
    place_digits(g, pass, blockIdx.x * g.tile, before, all, next, part);
}

// Fewer places are put in order by one launch that counts: a token's rank is the number of smaller ones and of equal ones before it.  A
// workgroup has kRankTile places, each wavefront all of them twice: its halves look through other blocks of 64 tokens, from LDS.  Without
// places: zeros only.  n^2 comparisons, bound by their instructions and LDS reads: 2,000 places 5.7 us, 8,000 10.0 (with 20 MB of zeros beside them
// 7.2 and 13.2; workgroups of 16 places 7.0 and 15.3); the passes above take 23 for 8,193, two of one workgroup 27 for 8,000.
constexpr uint32_t kRankPlaces = 8192, kRankTile = 32, kRankBlock = 64;

__global__ __launch_bounds__(kSortThreads) void rank_tokens_kernel(SortArgs g, uint32_t tiles, ClearArgs clear) {
    constexpr uint32_t kParts = kWave / kRankTile, kPitch = kRankBlock + 4;         // (the parts' reads in different banks)
    __shared__ __align__(16) uint32_t keys[kRankPlaces / kRankBlock * kPitch];
    __shared__ uint32_t ranks[kRankTile];
    if (blockIdx.x >= tiles) {
        clear_units(clear, blockIdx.x - tiles, gridDim.x - tiles);
        return;
    }
    const uint32_t tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const uint32_t blocks = (g.n + kRankBlock - 1) / kRankBlock;
    auto fill = [&](const auto* tokens) __attribute__((always_inline)) {    // (all of a thread's tokens on their way at once)
        int64_t v[kRankPlaces / kSortThreads];
#pragma unroll
        for (uint32_t u = 0; u < kRankPlaces / kSortThreads; ++u) v[u] = tokens[min(u * kSortThreads + tid, g.n - 1)];
#pragma unroll
        for (uint32_t u = 0; u < kRankPlaces / kSortThreads; ++u) {
            const uint32_t i = u * kSortThreads + tid;
            const uint32_t key = v[u] >= 0 && v[u] < (int64_t)g.V ? (uint32_t)v[u] : g.V;
            if (i < blocks * kRankBlock) keys[i / kRankBlock * kPitch + i % kRankBlock] = i < g.n ? key : ~0u;      // (past the last place: after all)
        }
    };
    if (g.wide_tokens) fill(static_cast<const int64_t*>(g.tokens));
    else fill(static_cast<const int32_t*>(g.tokens));
    if (tid < kRankTile) ranks[tid] = 0u;
    __syncthreads();
    const uint32_t i = blockIdx.x * kRankTile + lane % kRankTile, own = i / kRankBlock, mine = keys[own * kPitch + i % kRankBlock];
    uint32_t rank = 0;
    for (uint32_t b0 = wave * kParts; b0 < blocks; b0 += kSortWaves * kParts) {
        const uint32_t b = b0 + lane / kRankTile;
        if (b >= blocks) break;
        const uint32_t* block = keys + b * kPitch;
        auto count = [&](auto smaller) __attribute__((always_inline)) {
#pragma unroll
            for (uint32_t e = 0; e < kRankBlock; e += 4) {
                const uint4 k = *reinterpret_cast<const uint4*>(block + e);
                const uint32_t other[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) rank += smaller(other[u], e + u) ? 1u : 0u;
            }
        };
        const uint32_t below = mine + (b < own ? 1u : 0u);     // of the blocks before, equal ones count too
        if (own < b0 || own >= b0 + kParts) count([&](uint32_t other, uint32_t) { return other < below; });
        else count([&](uint32_t other, uint32_t at) { return other < (b == own && at < i % kRankBlock ? mine + 1u : below); });
    }
    atomicAdd(&ranks[lane % kRankTile], rank);
    __syncthreads();
    if (tid < kRankTile && i < g.n) {
        const uint32_t to = ranks[tid];
        g.key[0][to] = mine;
        g.place[0][to] = i;
    }
}

// ---- gradient: sums ----------------------------------------------------------------------------------------------------
constexpr int kSumThreads = 256;
constexpr int kSumE = 4;                   // columns of a lane: sums are mostly written as floats, 16 bytes a lane then
constexpr int kSumRows = 8;                // rows on their way at a time

struct SumArgs {
    const uint32_t* key;                   // n, ascending
    const uint32_t* place;
    const void* grad;
    void* out;
    float* parts;                          // chunks x 2 x D: of the token that began before the chunk, of the one that goes on after it
    uint32_t n, V, chunk;                  // chunk: places of a group
    uint32_t sections;                     // workgroups follow each other by chunk, then by section of columns
    int64_t D, grad_stride, out_stride;
    float scale;
    int log_lanes, accumulate, stream;
};

// the values of one lane: a piece, or of rows shorter than one the row's
template <int E>
struct Lane {
    WholePiece<E> at;
    int narrow;                            // values of such a row, else 0
    __device__ __forceinline__ Lane(int64_t col, int64_t D) : at(D < E ? 0 : col, D < E ? E : D), narrow(D < E ? (int)D : 0) {}
    template <typename T>
    __device__ __forceinline__ typename Piece_<T, E>::type load(const T* row) const { return narrow ? load_raw<T, E>(row, narrow) : at.template load<T>(row); }
    template <typename T>
    __device__ __forceinline__ void store(T* row, typename Floats<E>::type v, bool stream = false) const {
        if (narrow) store_piece<T, E>(row, v, narrow);
        else at.template store<T>(row, v, stream);
    }
};

template <typename TY, int E>
__device__ __forceinline__ void finish_row(const SumArgs& g, uint32_t v, const Lane<E>& lane, typename Floats<E>::type sum) {
    TY* dst = static_cast<TY*>(g.out) + (int64_t)v * g.out_stride;
    sum = sum * g.scale;
    if (g.accumulate) sum = sum + __builtin_convertvector(lane.template load<TY>(dst), typename Floats<E>::type);
    lane.template store<TY>(dst, sum, g.stream);
}

template <typename TX, typename TY>
__global__ __launch_bounds__(kSumThreads) void sum_rows_kernel(SumArgs g) {
    constexpr int E = kSumE;
    typedef typename Floats<E>::type F;
    const int tid = threadIdx.x;
    const int lanes = 1 << g.log_lanes, l = tid & (lanes - 1);
    const uint32_t block = blockIdx.x / g.sections, section = blockIdx.x - block * g.sections;
    const uint32_t c = block * (kSumThreads >> g.log_lanes) + (tid >> g.log_lanes);
    const uint64_t start = (uint64_t)c * g.chunk;
    const int64_t col = (((int64_t)section << g.log_lanes) + l) * E;
    if (start >= g.n || col >= g.D) return;
    const uint32_t j0 = (uint32_t)start, j1 = (uint32_t)min((uint64_t)g.n, start + g.chunk);
    const Lane<E> lane(col, g.D);
    const TX* grad = static_cast<const TX*>(g.grad);
    float* part = g.parts + (size_t)c * 2 * g.D;
    uint32_t cur = g.key[j0];
    bool from_before = j0 > 0 && g.key[j0 - 1] == cur;
    F sum;
    sum = 0.0f;
    // (no load stands behind a condition: what is past the chunk's end repeats its last row, which is not added)
    uint32_t key[kSumRows], place[kSumRows];
    auto look = [&](uint32_t j) {
#pragma unroll
        for (int u = 0; u < kSumRows; ++u) {
            const uint32_t at = min(j + u, j1 - 1);
            key[u] = g.key[at];
            place[u] = g.place[at];
        }
    };
    look(j0);
    for (uint32_t j = j0; j < j1; j += kSumRows) {
        typename Piece_<TX, E>::type r[kSumRows];
        uint32_t token[kSumRows];
#pragma unroll
        for (int u = 0; u < kSumRows; ++u) {
            r[u] = lane.template load<TX>(grad + (int64_t)place[u] * g.grad_stride);
            token[u] = key[u];
        }
        look(j + kSumRows);                                   // the next rows' places, while these rows are on their way
#pragma unroll
        for (int u = 0; u < kSumRows; ++u) {
            if (j + u < j1) {
                if (token[u] != cur) {
                    if (from_before) lane.template store<float>(part, sum);
                    else finish_row<TY, E>(g, cur, lane, sum);           // (cur < V: a larger token follows it, and V is the largest)
                    from_before = false;
                    cur = token[u];
                    sum = 0.0f;
                }
                if (cur < g.V) sum = sum + __builtin_convertvector(r[u], F);
            }
        }
    }
    if (cur >= g.V) return;
    const bool goes_on = j1 < g.n && g.key[j1] == cur;
    if (from_before) lane.template store<float>(part, sum);
    else if (goes_on) lane.template store<float>(part + g.D, sum);
    else finish_row<TY, E>(g, cur, lane, sum);
}

// Tokens that go on after the chunk they began in: a wavefront looks at the end of one chunk and adds up the token's parts if they
// are few; of those with more, the workgroup's four wavefronts take a quarter of the parts each.  2,048 chunks of 1,024 columns
// take 10.6 us, the chain of reads to a token's end and parts (a workgroup a chunk: 11.6, of 512 threads 17.5, for starting many that find nothing).
template <typename TY>
__global__ __launch_bounds__(kSumThreads) void join_kernel(SumArgs g) {
    constexpr int E = 4, kWaves = kSumThreads / kWave;
    __shared__ f32x4 sums[kWaves][kWave];
    __shared__ uint32_t many[kWaves];                          // parts of the wavefronts' tokens, where the workgroup adds them up
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t col = ((int64_t)blockIdx.y * kWave + lane) * E;
    const Lane<E> own(col < g.D ? col : 0, g.D);
    // parts lo .. hi - 1 of the token that began in chunk c: part 0 is chunk c's own, part i that of the i-th chunk after it
    auto add_parts = [&](uint32_t c, uint32_t lo, uint32_t hi) {
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t i = lo; i < hi; i += kSumRows) {
            typename Piece_<float, E>::type r[kSumRows];
#pragma unroll
            for (int u = 0; u < kSumRows; ++u) {
                const uint32_t at = min(i + u, hi - 1);
                r[u] = own.template load<float>(g.parts + ((size_t)(c + at) * 2 + (at == 0 ? 1 : 0)) * g.D);
            }
#pragma unroll
            for (int u = 0; u < kSumRows; ++u)
                if (i + u < hi) sum = sum + r[u];
        }
        return sum;
    };
    // how many parts the token that goes on after chunk c has, if it began there: one more than chunks after c begin with it
    auto parts_of = [&](uint32_t c, uint32_t& v) -> uint32_t {
        const uint64_t end = ((uint64_t)c + 1) * g.chunk;
        if (end >= g.n) return 0;
        const uint32_t j1 = (uint32_t)end, j0 = j1 - g.chunk;
        v = g.key[j1 - 1];
        const uint32_t after = g.key[j1], first = g.key[j0], before = g.key[max(j0, 1u) - 1u];
        if (v >= g.V || after != v) return 0;
        if (first == v && j0 > 0 && before == v) return 0;     // an earlier chunk's
        uint32_t parts = 1;
        while (true) {
            const uint64_t at = ((uint64_t)c + parts + lane) * g.chunk;
            const unsigned long long more = __ballot(at < g.n && g.key[min(at, (uint64_t)g.n - 1)] == v);
            const uint32_t run = more == ~0ull ? kWave : (uint32_t)__ffsll((long long)~more) - 1u;
            parts += run;
            if (run < kWave) return parts;
        }
    };
    const uint32_t c0 = blockIdx.x * kWaves;
    uint32_t v = 0;
    const uint32_t parts = parts_of(c0 + wave, v);
    if (lane == 0) many[wave] = parts > kSumRows ? parts : 0u;
    if (parts > 0 && parts <= kSumRows && col < g.D) finish_row<TY, E>(g, v, own, add_parts(c0 + wave, 0, parts));
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t all = many[w];
        if (all == 0) continue;                                // (the same for the workgroup)
        const uint32_t per = (all + kWaves - 1) / kWaves;
        f32x4 sum = add_parts(c0 + w, min(all, wave * per), min(all, (wave + 1) * per));
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == w && col < g.D) {
            sum = sums[0][lane];
#pragma unroll
            for (int o = 1; o < kWaves; ++o) sum = sum + sums[o][lane];
            finish_row<TY, E>(g, v, own, sum);
        }
        __syncthreads();
    }
}

// ---- gradient of few places --------------------------------------------------------------------------------------------
// Up to kFewPlaces places need no order: every workgroup looks through all the tokens by itself.  A workgroup for each place (and section of
// columns) sums its token's rows if no earlier place has it, its wavefronts a share of them each; workgroups behind those clear the
// rows that no token names.  One launch; the three with an order wait for memory a few times each, but start fewer wavefronts.  Measured (by one,
// by three): 300 places x 1,024 columns 6.9 and 15.2 us, 1,000 x 256 6.2 and 15.2, 1,000 x 1,024 14.8 and 16.0, 512 x 4,096 (8,192
// workgroups) 21.8 and 19.6, 1,000 x 4,096 47 and 20; 1,000 places of one token 21 and 14.
constexpr uint32_t kFewPlaces = 1024;      // two tokens a thread
constexpr int64_t kFewBlocks = 4096;       // workgroups for places and sections
constexpr int kFewClear = 8;               // table rows a wavefront clears

struct FewArgs {
    SumArgs sum;
    const void* tokens;
    int wide_tokens;
    uint32_t sum_blocks;
};

// NT: 256 threads for up to 512 places, 512 for more
template <typename TX, typename TY, int NT>
__global__ __launch_bounds__(NT) void few_places_kernel(FewArgs f) {
    constexpr int E = kSumE, kWaves = NT / kWave;
    const SumArgs& g = f.sum;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    int64_t mine[2];                                           // the tokens of places tid and NT + tid
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t i = h * NT + tid;
        mine[h] = token_at(f.tokens, f.wide_tokens, min(i, g.n - 1));
        if (i >= g.n) mine[h] = -1;
    }
    if (blockIdx.x >= f.sum_blocks) {
        constexpr int kClear = kFewClear * kWaves;
        __shared__ unsigned long long named;
        const int64_t v0 = (int64_t)(blockIdx.x - f.sum_blocks) * kClear;
        if (tid == 0) named = 0u;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (mine[h] >= v0 && mine[h] < v0 + kClear) atomicOr(&named, 1ull << (int)(mine[h] - v0));
        __syncthreads();
        for (int r = wave; r < kClear; r += kWaves) {
            if (((named >> r) & 1u) || v0 + r >= g.V) continue;
            TY* row = static_cast<TY*>(g.out) + (v0 + r) * g.out_stride;
            for (int64_t c = lane * E; c < g.D; c += kWave * E) store_piece<TY, E>(row + c, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, (int)min((int64_t)E, g.D - c));
        }
        return;
    }
    __shared__ uint32_t places[2 * NT];
    __shared__ uint32_t counts[2 * kWaves];
    __shared__ f32x4 sums[kWaves][kWave];
    const uint32_t t = blockIdx.x / g.sections, section = blockIdx.x - t * g.sections;
    const int64_t v = token_at(f.tokens, f.wide_tokens, t);
    if (v < 0 || v >= g.V) return;
    // the token's places in order
    unsigned long long same[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        same[h] = __ballot(mine[h] == v);
        if (lane == 0) counts[h * kWaves + wave] = (uint32_t)__popcll(same[h]);
    }
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t before = 0;
        for (int w = 0; w < 2 * kWaves; ++w) before += w < h * kWaves + wave ? counts[w] : 0u;
        if (mine[h] == v) places[before + (uint32_t)__popcll(same[h] & ((1ull << lane) - 1ull))] = h * NT + tid;
    }
    for (int w = 0; w < 2 * kWaves; ++w) total += counts[w];
    __syncthreads();
    if (places[0] != t) return;                                // an earlier place's workgroup has it
    const uint32_t per = (total + kWaves - 1) / kWaves, hi = min(total, (wave + 1) * per);
    const int64_t col = ((int64_t)section * kWave + lane) * E;
    const Lane<E> own(col < g.D ? col : 0, g.D);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t i = wave * per; i < hi; i += kSumRows) {
        typename Piece_<TX, E>::type r[kSumRows];
#pragma unroll
        for (int u = 0; u < kSumRows; ++u) r[u] = own.template load<TX>(static_cast<const TX*>(g.grad) + (int64_t)places[min(i + u, hi - 1)] * g.grad_stride);
#pragma unroll
        for (int u = 0; u < kSumRows; ++u)
            if (i + u < hi) sum = sum + __builtin_convertvector(r[u], f32x4);
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave || col >= g.D) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum = sum + sums[w][lane];
    finish_row<TY, E>(g, (uint32_t)v, own, sum);
}

// Places that few_places() takes use no workspace.  Above kNoWorkspace of them one is asked for all the same: how much room a number of
// places needs is part of the interface, and does not move with where one way turns out faster than the other.
constexpr int64_t kNoWorkspace = 512;
bool few_places(int64_t n, int64_t D) { return n <= kFewPlaces && n * ((D + kWave * kSumE - 1) / (kWave * kSumE)) <= kFewBlocks; }

// Places of a chunk: about 2,048 groups' worth, at least 16 so that few tokens are in parts, at most 256
uint32_t chunk_places(int64_t n) {
    uint32_t c = 16;
    while (c < 256 && (int64_t)c * 2048 < n) c *= 2;
    return c;
}

struct GradientSpace {                     // byte offsets of the workspace
    size_t key[2], place[2], counts, parts, total;
    uint32_t tile, tiles, chunk, chunks;
};
GradientSpace gradient_space(int64_t n, int64_t D) {
    GradientSpace s{};
    const int64_t least = n <= kRankPlaces ? n : std::max<int64_t>(kSortTile, (n + kSortTiles - 1) / kSortTiles);
    s.tile = (uint32_t)((least + kSortThreads - 1) / kSortThreads * kSortThreads);
    s.tiles = (uint32_t)((n + s.tile - 1) / s.tile);
    s.chunk = chunk_places(n);
    s.chunks = (uint32_t)((n + s.chunk - 1) / s.chunk);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t p = at; at += (bytes + 255) / 256 * 256; return p; };
    for (int i = 0; i < 2; ++i) s.key[i] = take(sizeof(uint32_t) * (size_t)n);
    for (int i = 0; i < 2; ++i) s.place[i] = take(sizeof(uint32_t) * (size_t)n);
    s.counts = take(sizeof(uint32_t) * (size_t)s.tiles * kSortBins);
    s.parts = take(sizeof(float) * 2 * (size_t)s.chunks * (size_t)D);
    s.total = at;
    return s;
}

int log_lanes_for(int64_t pieces) {
    int l = 0;
    while (l < 6 && ((int64_t)1 << l) < pieces) ++l;
    return l;
}

}  // namespace
}  // namespace pqt

extern "C" {

int pqt_embed(const void* table, int type, int64_t V, int64_t D, int64_t table_stride, const void* tokens, int token_bytes,
              int64_t n, float scale, void* out, int out_type, int64_t out_stride, int device, void* hip_stream) {
    using namespace pqt;
    if (!known_type(type) || !known_type(out_type)) return fail(PQT_EINVAL, "pqt_embed: unknown type %d or %d", type, out_type);
    if (token_bytes != 4 && token_bytes != 8) return fail(PQT_EINVAL, "pqt_embed: tokens of %d bytes (4 or 8)", token_bytes);
    if (V < 1 || D < 1 || n < 0 || table_stride < D || out_stride < D)
        return fail(PQT_EINVAL, "pqt_embed: V=%lld D=%lld n=%lld strides %lld, %lld out of range", (long long)V, (long long)D, (long long)n,
                    (long long)table_stride, (long long)out_stride);
    if (n == 0) return PQT_OK;
    if (!table || !tokens || !out) return fail(PQT_EINVAL, "pqt_embed: null pointer");
    if (!aligned_to(table, type_bytes(type)) || !aligned_to(out, type_bytes(out_type)) || !aligned_to(tokens, (size_t)token_bytes))
        return fail(PQT_EINVAL, "pqt_embed: a pointer is not aligned to its element");
    if (D > kMaxEmbedD) return fail(PQT_EUNSUPPORTED, "pqt_embed: D=%lld beyond 2^20", (long long)D);
    if (const int rc = check_device(device, "pqt_embed")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    const int E = type_bytes(type) == 2 && type_bytes(out_type) == 2 ? 8 : 4;
    EmbedArgs g{table, tokens, out, V, D, table_stride, n, out_stride, scale, log_lanes_for((D + E - 1) / E), token_bytes == 8,
                (double)n * D * type_bytes(out_type) > kStreamBytes};
    const int64_t pieces = (D + E - 1) / E, per_block = kEmbedThreads >> g.log_lanes;
    const int np = pieces <= 64 ? 1 : pieces <= 128 ? 2 : 4;
    const int64_t section = ((int64_t)np << g.log_lanes) * E;
    const dim3 grid((unsigned)std::min<int64_t>((n + per_block - 1) / per_block, kEmbedBlocks), (unsigned)((D + section - 1) / section));
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    with_type(type, [&](auto x) {
        with_type(out_type, [&](auto y) {
            using X = decltype(x);
            using Y = decltype(y);
            if (np == 1) hipLaunchKernelGGL((embed_kernel<X, Y, 1>), grid, dim3(kEmbedThreads), 0, st, g);
            else if (np == 2) hipLaunchKernelGGL((embed_kernel<X, Y, 2>), grid, dim3(kEmbedThreads), 0, st, g);
            else hipLaunchKernelGGL((embed_kernel<X, Y, 4>), grid, dim3(kEmbedThreads), 0, st, g);
        });
    });
    HIP_TRY(hipGetLastError());
    return PQT_OK;
}

size_t pqt_embed_gradient_workspace(int64_t n, int64_t V, int64_t D) {
    if (n < 1 || V < 1 || D < 1 || (n <= pqt::kNoWorkspace && pqt::few_places(n, D)) || n > pqt::kMaxPlaces || V > pqt::kMaxRows || D > pqt::kMaxEmbedD) return 0;
    return pqt::gradient_space(n, D).total;
}

int pqt_embed_gradient(const void* grad, int grad_type, int64_t grad_stride, const void* tokens, int token_bytes, int64_t n,
                       int64_t V, int64_t D, float scale, int accumulate, void* out, int out_type, int64_t out_stride,
                       void* workspace, size_t workspace_bytes, int device, void* hip_stream) {
    using namespace pqt;
    if (!known_type(grad_type) || !known_type(out_type)) return fail(PQT_EINVAL, "pqt_embed_gradient: unknown type %d or %d", grad_type, out_type);
    if (token_bytes != 4 && token_bytes != 8) return fail(PQT_EINVAL, "pqt_embed_gradient: tokens of %d bytes (4 or 8)", token_bytes);
    if (V < 1 || D < 1 || n < 0 || grad_stride < D || out_stride < D)
        return fail(PQT_EINVAL, "pqt_embed_gradient: V=%lld D=%lld n=%lld strides %lld, %lld out of range", (long long)V, (long long)D,
                    (long long)n, (long long)grad_stride, (long long)out_stride);
    if (n > kMaxPlaces || V > kMaxRows || D > kMaxEmbedD)
        return fail(PQT_EUNSUPPORTED, "pqt_embed_gradient: n=%lld V=%lld D=%lld beyond the limits", (long long)n, (long long)V, (long long)D);
    if (!out || (n > 0 && (!grad || !tokens))) return fail(PQT_EINVAL, "pqt_embed_gradient: null pointer");
    if (!aligned_to(grad, type_bytes(grad_type)) || !aligned_to(out, type_bytes(out_type)) || !aligned_to(tokens, (size_t)token_bytes))
        return fail(PQT_EINVAL, "pqt_embed_gradient: a pointer is not aligned to its element");
    const GradientSpace s = n > 0 && (n > kNoWorkspace || !few_places(n, D)) ? gradient_space(n, D) : GradientSpace{};
    if (s.total && (!workspace || workspace_bytes < s.total || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_embed_gradient: workspace of %zu bytes, aligned to 16, needed (%zu given)", s.total, workspace_bytes);
    const int log_lanes = log_lanes_for((D + kSumE - 1) / kSumE);
    const uint32_t groups = kSumThreads >> log_lanes;
    const int64_t section = (int64_t)kSumE << log_lanes, sections = (D + section - 1) / section, work = (s.chunks + groups - 1) / groups * sections;
    if (work > 0xffffff) return fail(PQT_EUNSUPPORTED, "pqt_embed_gradient: n=%lld D=%lld together beyond the grid", (long long)n, (long long)D);
    if (n == 0 && accumulate) return PQT_OK;
    if (const int rc = check_device(device, "pqt_embed_gradient")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    SumArgs g{};
    g.grad = grad;
    g.out = out;
    g.n = (uint32_t)n;
    g.V = (uint32_t)V;
    g.D = D;
    g.grad_stride = grad_stride;
    g.out_stride = out_stride;
    g.scale = scale;
    g.accumulate = accumulate != 0;
    g.stream = (double)V * D * type_bytes(out_type) > kStreamBytes;
    if (n > 0 && few_places(n, D)) {
        FewArgs f{g, tokens, token_bytes == 8, 0};
        f.sum.sections = (uint32_t)((D + kWave * kSumE - 1) / (kWave * kSumE));
        f.sum_blocks = (uint32_t)n * f.sum.sections;
        const int threads = n <= 512 ? 256 : 512, rows = kFewClear * (threads / kWave);
        const uint32_t clear = accumulate ? 0u : (uint32_t)((V + rows - 1) / rows);
        with_type(grad_type, [&](auto x) {
            with_type(out_type, [&](auto y) {
                if (threads == 256) hipLaunchKernelGGL((few_places_kernel<decltype(x), decltype(y), 256>), dim3(f.sum_blocks + clear), dim3(256), 0, st, f);
                else hipLaunchKernelGGL((few_places_kernel<decltype(x), decltype(y), 512>), dim3(f.sum_blocks + clear), dim3(512), 0, st, f);
            });
        });
        HIP_TRY(hipGetLastError());
        return PQT_OK;
    }
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    SortArgs o{};
    o.tokens = tokens;
    o.wide_tokens = token_bytes == 8;
    o.n = (uint32_t)n;
    o.V = (uint32_t)V;
    o.tile = s.tile;
    for (int i = 0; i < 2; ++i) {
        o.key[i] = reinterpret_cast<uint32_t*>(ws + s.key[i]);
        o.place[i] = reinterpret_cast<uint32_t*>(ws + s.place[i]);
    }
    o.counts = reinterpret_cast<uint32_t*>(ws + s.counts);
    int bits = 1;
    while (bits < 32 && ((uint64_t)V >> bits) != 0) ++bits;                 // V itself is a key
    o.passes = (bits + kSortBits - 1) / kSortBits;
    o.bits = (bits + o.passes - 1) / o.passes;
    // the zeros, in shares as long as the launches they go with take: a pass's counting one part, its placing two
    const int64_t row = D * (int64_t)type_bytes(out_type), step = out_stride * (int64_t)type_bytes(out_type);
    ClearArgs clear{};
    clear.out = static_cast<unsigned char*>(out);
    clear.total = V * row;
    clear.unit = row == step ? kClearUnit : row;
    clear.step = row == step ? kClearUnit : step;
    clear.stream = g.stream;
    const int64_t units = accumulate ? 0 : (clear.total + clear.unit - 1) / clear.unit;
    int part = 0;
    const int parts = s.tiles <= 1 ? 1 : 3 * o.passes;
    auto share = [&](int of) {                                              // the next `of` parts; returns their workgroups
        clear.first = units / parts * part + std::min<int64_t>(part, units % parts);
        part += of;
        clear.last = units / parts * part + std::min<int64_t>(part, units % parts);
        return (uint32_t)std::min<int64_t>((clear.last - clear.first + kSortWaves - 1) / kSortWaves, kClearBlocks);
    };
    if (s.tiles <= 1) {
        const uint32_t more = share(1), blocks = (uint32_t)((n + kRankTile - 1) / kRankTile);
        hipLaunchKernelGGL(rank_tokens_kernel, dim3(blocks + more), dim3(kSortThreads), 0, st, o, blocks, clear);
        HIP_TRY(hipGetLastError());
    } else {
        for (int pass = 0; pass < o.passes; ++pass) {
            uint32_t more = share(1);
            hipLaunchKernelGGL(token_counts_kernel, dim3(s.tiles + more), dim3(kSortThreads), 0, st, o, pass, s.tiles, clear);
            HIP_TRY(hipGetLastError());
            more = share(2);
            hipLaunchKernelGGL(token_places_kernel, dim3(s.tiles + more), dim3(kSortThreads), 0, st, o, pass, s.tiles, clear);
            HIP_TRY(hipGetLastError());
        }
    }
    if (n == 0) return PQT_OK;
    const int last = s.tiles <= 1 ? 0 : (o.passes - 1) & 1;
    g.key = o.key[last];
    g.place = o.place[last];
    g.parts = reinterpret_cast<float*>(ws + s.parts);
    g.chunk = s.chunk;
    g.sections = (uint32_t)sections;
    g.log_lanes = log_lanes;
    const dim3 grid((unsigned)work);
    with_type(grad_type, [&](auto x) {
        with_type(out_type, [&](auto y) {
            hipLaunchKernelGGL((sum_rows_kernel<decltype(x), decltype(y)>), grid, dim3(kSumThreads), 0, st, g);
        });
    });
    HIP_TRY(hipGetLastError());
    if (s.chunks > 1) {
        const dim3 join((s.chunks - 1 + kSumThreads / kWave - 1) / (kSumThreads / kWave), (unsigned)((D + 4 * kWave - 1) / (4 * kWave)));
        with_type(out_type, [&](auto y) { hipLaunchKernelGGL((join_kernel<decltype(y)>), join, dim3(kSumThreads), 0, st, g); });
        HIP_TRY(hipGetLastError());
    }
    return PQT_OK;
}

}  // extern "C"
