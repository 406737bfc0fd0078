// What attention and its gradient share (attention.hip, attention_gradient.hip): fragments and the matrix instructions, tiles of rows in LDS, which
// rows a workgroup has, and the bias by distance.
//
// Everything is built on products of 16 x 16 results over 32 values.  A fragment holds, of one of 16 rows (lane & 15), eight values: those of
// places 8 * (lane >> 4) .. + 7.  A result has its column in lane & 15 and rows 4 * (lane >> 4) .. + 3 in four registers.  So the results of two products
// that lie 16 rows apart are, column by column, a fragment of 32 places in the order place(e) = 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3): weights go
// from one product into the next without leaving their lane, if the other operand's values are taken in that order.
#pragma once
#include <algorithm>
#include <type_traits>

#include "encoder.hpp"
#include "text_rows.hpp"

namespace pqt {

struct AttentionArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* grad;
    const void* out_in;                    // gradient: what the forward pass wrote
    const float* lse_in;
    const void* starts;
    const void* lengths;                   // or null: texts reach to the next one
    const float* bias;                     // heads x buckets, or null
    const int32_t* distances;              // buckets of -reach .. reach
    void* out;
    float* lse;
    void* dq;
    void* dk;
    void* dv;
    float* delta;                          // heads x n
    float2* large_sums;                    // heads x n: of rows with a large sum (large_sum()), maximum and logarithm of the sum beside it
    float* parts;                          // workgroups x distances -reach .. reach
    float* key_parts;                      // splits x heads of keys x n x (dk, dv), where the queries of a key are shared out
    int64_t q_stride, k_stride, v_stride, grad_stride, out_stride, dq_stride, dk_stride, dv_stride;
    int64_t n, texts;
    int64_t tiles;                         // workgroups of a head
    int wide;                              // starts and lengths are 64-bit numbers
    int heads, group, d, buckets, reach, clear;
    float scale, inverse_scale;
};

// The kernels are compiled for one type in a translation unit of its own (attention_bf16.hip and so on): their launchers, by the rows of a workgroup
// (16, 64 or 128), for rows that direct_rows() holds of or any.
template <typename T> void launch_attention(const AttentionArgs& g, int rows, bool direct, hipStream_t st);
template <typename T> void launch_attention_queries(const AttentionArgs& g, int rows, bool direct, hipStream_t st);
template <typename T> void launch_attention_keys(const AttentionArgs& g, int rows, int splits, bool direct, hipStream_t st);

namespace {

constexpr int kMaxHeadD = 128;
constexpr int kMaxReach = 448;              // (the sums by distance of four wavefronts, 16 each, and the tiles of the widest heads fill LDS)
constexpr int kMaxBuckets = 1024;
constexpr int64_t kMaxRows = 0x7ffffff0;       // rows of a text are 32-bit numbers
constexpr int64_t kMaxWorkgroups = 0xffffff;   // of up to 256 threads each, fewer than 2^32 in all
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLog2eRest = (float)(1.44269504088896340736 - (double)kLog2e);

// ---- fragments -------------------------------------------------------------------------------------------------------
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct FragmentOf;
template <> struct FragmentOf<Bf16> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
    typedef u32x4 piece __attribute__((aligned(2)));           // 16 bytes at any element
};
template <> struct FragmentOf<Half> {
    typedef _Float16 type __attribute__((ext_vector_type(8)));
    typedef u32x4 piece __attribute__((aligned(2)));
};
template <> struct FragmentOf<float> {
    typedef float type __attribute__((ext_vector_type(8)));
    typedef u32x4 piece __attribute__((aligned(4)));
};
template <typename T> struct Stored { typedef T type; };
template <> struct Stored<Bf16> { typedef __bf16 type; };
template <> struct Stored<Half> { typedef _Float16 type; };
template <typename T> using Fragment = typename FragmentOf<T>::type;

__device__ __forceinline__ f32x4 multiply(Fragment<Bf16> a, Fragment<Bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(Fragment<Half> a, Fragment<Half> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// fp32: eight instructions over four places each, the e-th over the e-th values of the four groups of lanes
__device__ __forceinline__ f32x4 multiply(Fragment<float> a, Fragment<float> b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// results of two products 16 rows apart as a fragment (rounded to nearest even)
template <typename T>
__device__ __forceinline__ Fragment<T> fragment_of(f32x4 lo, f32x4 hi) {
    f32x8 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = lo[e];
        v[e + 4] = hi[e];
    }
    return __builtin_convertvector(v, Fragment<T>);
}

// ---- tiles of rows in LDS --------------------------------------------------------------------------------------------
// ROWS rows of DP values in pieces of 16 bytes, which lie permuted by the row's number, so that the rows whose pieces are read together fall into different
// banks (the lanes that a 16-byte read serves together are 0-3, 12-15, 20-27 and so on: see the rows of a fragment).
template <typename T, int ROWS, int DP>
struct Tile {
    typedef typename Stored<T>::type S;
    typedef __attribute__((address_space(3))) S* Place;
    static constexpr int E = 16 / (int)sizeof(T), kOfRow = DP / E, kSize = ROWS * DP;
    Place v;                               // an LDS array of kSize values
    int lane;                              // of the wavefront

    static __device__ __forceinline__ int turn(int row) { return kOfRow % 16 == 0 ? row & 15 : kOfRow % 8 == 0 ? row & 7 : row & 8 ? 3 : 0; }
    // values 32 chunk + 8 (lane >> 4) .. + 7 of row row0 + (lane & 15)
    __device__ __forceinline__ Fragment<T> rows(int row0, int chunk) const {
        const int row = lane & 15, q = lane >> 4;
        const Place p = v + (row0 + row) * DP;
        typedef __attribute__((address_space(3))) const u32x4 P;
        if constexpr (sizeof(T) == 2) {
            return __builtin_bit_cast(Fragment<T>, *(P*)(p + ((chunk * 4 + q) ^ turn(row)) * E));
        } else {
            const u32x4 lo = *(P*)(p + ((chunk * 8 + q * 2) ^ turn(row)) * E), hi = *(P*)(p + ((chunk * 8 + q * 2 + 1) ^ turn(row)) * E);
            return __builtin_shufflevector(__builtin_bit_cast(f32x4, lo), __builtin_bit_cast(f32x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // the transpose's: of column 16 block + (lane & 15), the rows row0 + place(e)
    __device__ __forceinline__ Fragment<T> columns(int row0, int block) const {
        const int col = lane & 15, q = lane >> 4;
        if constexpr (sizeof(T) == 2) {
            // sixteen lanes read 4 x 16 values, 8 bytes each, and get a column's four
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int row = q * 4 + (col >> 2);
            const Place p = v + (row0 + row) * DP + (((block * 2 + ((col >> 1) & 1)) ^ turn(row)) * E + (col & 1) * 4);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * DP));
            return __builtin_bit_cast(Fragment<T>, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            Fragment<T> f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = q * 4 + (e & 3);
                f[e] = v[(row0 + 16 * (e >> 2) + row) * DP + ((block * 4 + (col >> 2)) ^ turn(row)) * E + (col & 3)];
            }
            return f;
        }
    }
};

// What brings ROWS rows of d values, from row0 on, of the `len` at base to a tile, zeros in rows past len and in values past d: begin(), other work, finish(),
// and a barrier.
// DIRECT: straight to LDS, 16 bytes a lane; rows begin at multiples of 16 bytes and are whole pieces, and a tile spans less than 2^31 bytes (direct_rows()).
// Else by registers; rows begin anywhere, and their last piece is read value by value.
template <typename T, int ROWS, int DP, int THREADS, bool DIRECT>
struct Loader {
    typedef Tile<T, ROWS, DP> Into;
    static constexpr int E = Into::E, kOfRow = Into::kOfRow, kPieces = ROWS * kOfRow / THREADS;
    static_assert(ROWS * kOfRow % THREADS == 0, "whole pieces for every thread");
    static constexpr uint32_t kNowhere = 0x80000000u;
    typedef typename FragmentOf<T>::piece Unaligned;
    // where a thread's pieces lie equally far apart, the first one's place is kept, and the others' are counted from it
    static constexpr int kRowsApart = THREADS / kOfRow;
    static constexpr bool kEven = THREADS % kOfRow == 0 && kRowsApart % 16 == 0;
    u32x4 v[DIRECT ? 1 : kPieces];
    uint32_t off[DIRECT && !kEven ? kPieces : 1];

    __device__ __forceinline__ Loader(int64_t stride, int d) {
        if constexpr (DIRECT) {
#pragma unroll
            for (int i = 0; i < (kEven ? 1 : kPieces); ++i) {
                const int at = threadIdx.x % THREADS + i * THREADS, row = at / kOfRow, c = ((at % kOfRow) ^ Into::turn(row)) * E;
                off[i] = c < d ? (uint32_t)((row * (int)stride + c) * (int)sizeof(T)) : kNowhere;
            }
        }
    }
    __device__ __forceinline__ void begin(Into tile, const T* base, int64_t stride, int row0, int len, int d) {
        if constexpr (DIRECT) {
            typedef __attribute__((address_space(3))) void lds_bytes;
            const uint64_t at = (uint64_t)(base + (int64_t)row0 * stride);
            const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
            const int rows = min(len - row0, ROWS);
            const uint32_t bytes = __builtin_amdgcn_readfirstlane((uint32_t)(((rows - 1) * (int)stride + d) * (int)sizeof(T)));
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), (short)0, bytes, 0x00027000);
            const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x % THREADS) / kWave);
            const uint32_t apart = kRowsApart * (uint32_t)stride * (uint32_t)sizeof(T);    // (kNowhere stays past every tile)
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#if defined(__HIP_DEVICE_COMPILE__)                            // (the host's pass over this file takes 16 bytes for an error, and leaves the kernels out)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_bytes*)(tile.v + (i * THREADS + wave * kWave) * E), 16, kEven ? off[0] + i * apart : off[i], 0, 0, 0);
#else
                (void)from, (void)wave, (void)apart;
#endif
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int at = threadIdx.x % THREADS + i * THREADS, row = row0 + at / kOfRow, c = ((at % kOfRow) ^ Into::turn(at / kOfRow)) * E;
                v[i] = u32x4{};
                if (row < len && c < d) v[i] = piece(base + (int64_t)row * stride + c, d - c);
            }
        }
    }
    __device__ __forceinline__ void finish(Into tile) {
        if constexpr (DIRECT) __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0)
        else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) *(__attribute__((address_space(3))) u32x4*)(tile.v + (threadIdx.x % THREADS + i * THREADS) * E) = v[i];
        }
    }
    static __device__ __forceinline__ u32x4 piece(const T* p, int have) {
        if (have >= E) return *reinterpret_cast<const Unaligned*>(p);
        union { u32x4 v; T e[E]; } u;
        u.v = u32x4{};
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j < have) u.e[j] = p[j];
        return u.v;
    }
};
inline bool direct_rows(const void* p, int64_t stride, size_t element, int d) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * element % 16 == 0 && d * element % 16 == 0 && stride * (int64_t)element < (1 << 24);
}

// fragment `chunk` of a wavefront's own 16 rows row0 + (lane & 15), straight from memory
template <typename T>
__device__ __forceinline__ Fragment<T> rows_of_memory(const T* base, int64_t stride, int row0, int len, int d, int chunk, int lane) {
    const int row = row0 + (lane & 15), c = chunk * 32 + (lane >> 4) * 8;
    typedef typename Piece_<T, 8>::type V;
    V v = V{};
    if (row < len && c < d) v = load_raw<T, 8>(base + (int64_t)row * stride + c, d - c);
    return __builtin_bit_cast(Fragment<T>, v);
}

// The same where rows are whole aligned pieces, of the rows at base from 0 to last, without a branch and with the lanes' places in 32 bits: a row past the
// last is read as that, and it is the caller who leaves it out.
template <typename T>
__device__ __forceinline__ Fragment<T> whole_rows_of_memory(const T* base, uint32_t stride_bytes, int row0, int last, int d, int chunk, int lane) {
    const int c = chunk * 32 + (lane >> 4) * 8;
    const uint32_t row = (uint32_t)min(row0 + (lane & 15), last) * stride_bytes;
    const char* p = reinterpret_cast<const char*>(base);
    constexpr int E = 16 / (int)sizeof(T);
    u32x4 v[8 / E];
#pragma unroll
    for (int i = 0; i < 8 / E; ++i) {
        v[i] = *reinterpret_cast<const u32x4*>(p + (row + (uint32_t)min(c + i * E, d - E) * (uint32_t)sizeof(T)));
        if (chunk * 32 + 32 > d && c + i * E >= d) v[i] = u32x4{};
    }
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(Fragment<T>, v[0]);
    else return __builtin_shufflevector(__builtin_bit_cast(f32x4, v[0]), __builtin_bit_cast(f32x4, v[1]), 0, 1, 2, 3, 4, 5, 6, 7);
}

// ---- which rows ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ int64_t number(const void* p, int wide, int64_t i) {
    return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
}

// The lanes of a wavefront, of which each sees a text's start.
struct Looking {
    const AttentionArgs& g;
    int probe, seen;
    int64_t held;

    __device__ __forceinline__ int in_range(int64_t start) const { return (int)min(max(start, (int64_t)0), g.n); }
    __device__ __forceinline__ void look(int lo, int step) {
        const int texts = (int)g.texts;
        probe = lo + (int)(threadIdx.x & (kWave - 1)) * step;
        const int s = min(probe, texts);
        seen = in_range(number(g.starts, g.wide, s));
        held = 0;                                              // (asked for beside the starts of the last look, not behind them)
        if (step == 1 && g.lengths && texts) held = number(g.lengths, g.wide, min(s, texts - 1));
    }
    template <int M>
    __device__ __forceinline__ int count(int hi, int64_t t) const { return (int)__popcll(__ballot(probe < hi && seen / M + probe <= t)); }
    __device__ __forceinline__ int start(int lane) const { return __builtin_amdgcn_readlane(seen, lane); }
    __device__ __forceinline__ int start_of(int text) const { return __builtin_amdgcn_readfirstlane(in_range(number(g.starts, g.wide, text))); }
    __device__ __forceinline__ int tokens(int lane) const { return __builtin_amdgcn_readlane((int)min(max(held, (int64_t)0), (int64_t)0x7fffffff), lane); }
};
template <int M>
__device__ __forceinline__ Rows rows_of_workgroup(const AttentionArgs& g, int64_t t) {
    Looking looking{g, 0, 0, 0};
    return rows_of_looks<M>(looking, g.n, (int)g.texts, g.lengths != nullptr, g.clear != 0, t);
}

// Where every second workgroup has no rows -- texts of exactly M, or of half of M -- the busy ones would all go to the same half of an XCD's shader engines,
// which get workgroups in turn: of every sixteen, the second four are swapped in pairs, the third in halves, the fourth turned round.  (512 texts of 128 tokens,
// 16 heads, 128 rows a workgroup: 232 us, 153 so; the gradient 894, 565.)  Longer texts, of whose workgroups two of three have rows, stay in order: a text of 8,191, 515 us so and 506.
__device__ __forceinline__ int64_t out_of_step(const AttentionArgs& g, int64_t t) { return g.tiles <= 3 * g.texts && (t | 3) < g.tiles ? t ^ (t >> 2 & 3) : t; }

// Workgroup -> (rows, head).  Consecutive workgroups go to the eight XCDs in turn: each XCD gets a run of one head's rows after another, so that its L2
// holds the keys and values that they share.
__device__ __forceinline__ void place_of_workgroup(const AttentionArgs& g, int heads, int64_t& t, int& head) {
    const int64_t total = g.tiles * heads, per = total >> 3;
    const int x = blockIdx.x & 7, more = (int)(total & 7);
    const int64_t at = x * per + min(x, more) + (blockIdx.x >> 3);
    head = (int)(at / g.tiles);
    t = out_of_step(g, at - (int64_t)head * g.tiles);
}

// The same where a row's heads are cut into `parts`, side by side.
__device__ __forceinline__ void place_of_part(const AttentionArgs& g, int parts, int64_t& t, int& part) {
    const int64_t total = g.tiles * parts, per = total >> 3;
    const int x = blockIdx.x & 7, more = (int)(total & 7);
    const int64_t at = x * per + min(x, more) + (blockIdx.x >> 3);
    t = at / parts;
    part = (int)(at - t * parts);
    t = out_of_step(g, t);
}

// Lanes of a wavefront meet: what one wrote to LDS another may read, in program order.
__device__ __forceinline__ void wave_meets() {
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");       // (loads to LDS may overwrite what is read by then)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// zeros in rows from .. to of d columns
template <typename T>
__device__ __forceinline__ void clear_rows(T* p, int64_t stride, int64_t from, int64_t to, int d) {
    for (int64_t e = threadIdx.x; e < (to - from) * d; e += blockDim.x) p[(from + e / d) * stride + e % d] = from_float<T>(0.0f);
}

// ---- the bias by distance --------------------------------------------------------------------------------------------
// Products are taken unscaled, with bias / scale as what they are added to, so that a logit is one multiplication by scale * log2 e away from its power
// of two.  Finite entries are kept within 2^90, where that multiplication (scale up to 2^32) cannot overflow; -inf stays.
constexpr float kBiasTop = 0x1p90f, kLowest = -0x1.fffffep127f;        // (kLowest: no finite logit is below)

__device__ __forceinline__ float scaled_bias(float entry, float inverse_scale) {
    const float v = entry * inverse_scale;
    return fabsf(entry) < __builtin_inff() ? fmaxf(-kBiasTop, fminf(v, kBiasTop)) : v;
}
// The bias of the distances on either side in LDS, four times, copy c shifted by c places: the four consecutive ones that a lane needs for a
// result then begin at a multiple of 16 bytes in copy (first & 3), which is the same for all of a lane's.
struct BiasTable {
    float* v;
    int pitch;
    static __host__ __device__ __forceinline__ int pitch_of(int most) { return (2 * most + 4 + 63) / 64 * 64 + 16; }      // for W up to `most`
    static size_t bytes(int most) { return 4 * sizeof(float) * pitch_of(most); }

    // In two parts, so that a workgroup can ask for the buckets before it knows its rows: for the distances -W .. W (SIGN -1: W .. -W) ...
    template <int SIGN, int THREADS, int N>
    static __device__ __forceinline__ void look_up(const AttentionArgs& g, int W, int (&bucket)[N]) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int i = threadIdx.x % THREADS + n * THREADS;
            bucket[n] = -1;
            if (n * THREADS <= 2 * W && i <= 2 * W) bucket[n] = g.distances[max(-g.reach, min(SIGN * (i - W), g.reach)) + g.reach];
        }
    }
    // ... and a head's bias of them, and of the two ends: of the distances up to S, which a short text does not pass
    template <int THREADS, int N>
    __device__ __forceinline__ void fill(const AttentionArgs& g, int head, int W, int S, const int (&bucket)[N]) const {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int i = threadIdx.x % THREADS + n * THREADS;
            if (n * THREADS > W + S || i < W - S || i > W + S) continue;
            const float b = (unsigned)bucket[n] < (unsigned)g.buckets ? scaled_bias(g.bias[(int64_t)head * g.buckets + bucket[n]], g.inverse_scale) : 0.0f;     // (no bucket: no bias)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (i >= c) v[c * pitch + i - c] = b;
        }
    }
    // where a lane finds places first, first + 1 .. (of which it reads four from multiples of four on)
    __device__ __forceinline__ const float* from(int first) const { return v + (first & 3) * pitch + (first & ~3); }
};
__device__ __forceinline__ f32x4 four_of(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// From this power of two on -- of a row's maximum, or of the sum that lse is the logarithm of -- a multiplication's rounding shows in the weights taken from it: 2^12 is
// up to 2^-12 off, a part in 6,000 of a weight, and a bias of -1e9 is 64 away from the next number.  Weights are taken from differences there.
constexpr float kLargePower = 0x1p12f;

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// the largest, and the sum, over the four groups of sixteen lanes
__device__ __forceinline__ float max_of_groups(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float sum_of_groups(float v) {
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}

// Kinds of steps along a text, a body each: all places farther than `reach` on one side (or no bias), some nearer, either of them, and the last, whose rows behind
// the text's end are left out.  (The gradient's second walk, for rows with a large sum, has one body for all.)
enum : int { kFar, kNear, kEither, kLast, kLarge };
template <int K> using Kind = std::integral_constant<int, K>;

// Steps of BN rows along a text of `len`, by a wavefront with 16 RT rows from row0 on, in turn by one of two tiles: f(kind, odd, step).  Every wavefront of a
// workgroup makes as many steps.  The last stands outside of the loop: what it alone needs takes no registers there.  RUNS: those far before the rows, those
// nearer than `reach` and those far behind are runs of their own (a choice at every step would move the sums from registers to others where its ways
// join, and what the products are added to as well); it takes code and registers that only long texts are worth.
template <int RT, int BN, bool RUNS, typename F>
__device__ __forceinline__ void walk(const AttentionArgs& g, int row0, int len, F&& f) {
    typedef std::integral_constant<bool, false> Even;
    typedef std::integral_constant<bool, true> Odd;
    const int full = (len - 1) / BN;
    int i = 0;
    if constexpr (!RUNS) {
        for (;; ++i) {
            if (i == full) break;
            f(Kind<kEither>{}, Even{}, i++);
            if (i == full) break;
            f(Kind<kEither>{}, Odd{}, i);
        }
    } else {
        // near: from the first j0 > row0 - reach - BN + 1 to the last j0 < row0 + 16 RT - 1 + reach
        const int near_from = g.bias ? min(full, (max(0, row0 - g.reach - BN + 2) + BN - 1) / BN) : full;
        const int near_to = g.bias ? min(full, (row0 + RT * 16 - 1 + g.reach + BN - 1) / BN) : full;
        auto run = [&](auto kind, int to) __attribute__((always_inline)) {
            if (i < to && i % 2) f(kind, Odd{}, i++);
#pragma nounroll
            for (; i + 1 < to; i += 2) {
                f(kind, Even{}, i);
                f(kind, Odd{}, i + 1);
            }
            if (i < to) f(kind, Even{}, i++);
        };
#pragma nounroll
        for (int side = 0; side < 2; ++side) {
            run(Kind<kFar>{}, side ? full : near_from);
            if (side == 0) run(Kind<kNear>{}, near_to);
        }
    }
    if (full % 2) f(Kind<kLast>{}, Odd{}, full);
    else f(Kind<kLast>{}, Even{}, full);
}

// calls f(Int<DP>) for heads of d values
template <int V> struct Width { static constexpr int value = V; };
template <typename F>
void with_head(int d, F&& f) {
    if (d <= 32) f(Width<32>{});
    else if (d <= 64) f(Width<64>{});
    else if (d <= 96) f(Width<96>{});
    else f(Width<128>{});
}

// ---- checks of the C entries, and the choice of workgroup -------------------------------------------------------------
inline int attention_checks(const char* who, int type, int64_t n, int heads, int kv_heads, int d, const void* starts, const void* lengths, int place_bytes,
                            int64_t texts, float scale, const float* bias, int buckets, const int32_t* distances, int reach, AttentionArgs& g) {
    using pqt_host::fail;
    if (!known_type(type)) return fail(PQT_EINVAL, "%s: unknown type %d", who, type);
    if (n < 0 || texts < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || d < 1)
        return fail(PQT_EINVAL, "%s: n=%lld texts=%lld heads=%d (of keys %d) d=%d out of range", who, (long long)n, (long long)texts, heads, kv_heads, d);
    if (place_bytes != 4 && place_bytes != 8) return fail(PQT_EINVAL, "%s: starts of %d bytes", who, place_bytes);
    if (!(scale >= 0x1p-32f && scale <= 0x1p32f)) return fail(PQT_EINVAL, "%s: scale=%g is not between 2^-32 and 2^32", who, (double)scale);
    if (bias && (buckets < 1 || reach < 0 || !distances)) return fail(PQT_EINVAL, "%s: a bias of %d buckets and distances up to %d", who, buckets, reach);
    if (n > 0 && !starts) return fail(PQT_EINVAL, "%s: null pointer", who);
    if (!aligned_to(starts, place_bytes) || !aligned_to(lengths, place_bytes) || !aligned_to(bias, 4) || !aligned_to(distances, 4))
        return fail(PQT_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (d > kMaxHeadD) return fail(PQT_EUNSUPPORTED, "%s: heads of %d values, at most %d", who, d, kMaxHeadD);
    if (bias && (buckets > kMaxBuckets || reach > kMaxReach))
        return fail(PQT_EUNSUPPORTED, "%s: %d buckets, at most %d; distances up to %d, at most %d", who, buckets, kMaxBuckets, reach, kMaxReach);
    if (n > kMaxRows || texts > kMaxRows || heads > 65535 || (n / 16 + texts + 1) * heads > kMaxWorkgroups)
        return fail(PQT_EUNSUPPORTED, "%s: %lld rows in %lld texts of %d heads", who, (long long)n, (long long)texts, heads);
    g.n = n;
    g.texts = texts;
    g.heads = heads;
    g.group = heads / kv_heads;
    g.d = d;
    g.starts = starts;
    g.lengths = lengths;
    g.wide = place_bytes == 8;
    g.scale = scale;
    g.inverse_scale = 1.0f / scale;
    g.bias = bias;
    g.buckets = buckets;
    g.distances = distances;
    g.reach = reach;
    return PQT_OK;
}

// Texts whose keys a wavefront takes without a workgroup's help.  (65,000 tokens or so, 16 heads of 64 bf16 values, this kernel and 64 rows a workgroup of the other: texts of
// 20 tokens 142 and 304 us, 36 203 and 215, 48 182 and 191, 64 191 and 167.)
inline bool short_texts(int64_t n, int64_t texts) { return texts > 0 && n / texts <= 48; }
// Heads that a wavefront takes one after the other: 16,384 wavefronts are two rounds of what the card holds.  (4,096 texts of 20 tokens, 16 heads: one head a
// wavefront 264 us, two 213, four 191.)  All wavefronts of a row get as many, or one fewer.
inline int heads_of_a_wavefront(int64_t tiles, int heads, int waves) {
    const int most = (int)std::max<int64_t>(1, std::min<int64_t>((heads + waves - 1) / waves, tiles * heads / 16384));
    const int parts = (heads + waves * most - 1) / (waves * most);
    return (heads + waves * parts - 1) / (waves * parts);
}

// Rows of a workgroup where texts are no short ones: wavefronts of two times 16 read a tile half as often, and 128 rows of a text of 64 or less would leave half of the workgroup
// without any.  (16 heads of 64 bf16 values, 64 and 128 rows, the gradient in brackets: 1,024 texts of 64 tokens 167 and 187 us (635, 749), 800 of 80 206 and 186
// (857, 775), 512 of 128 168 and 153 (662, 565).  Few workgroups: one text of 2,000 33 and 44 (112, 140), 2,500 49 and 53 (177, 184), 4,000 97 and 82 (367, 273).)
inline int rows_of_a_workgroup(int64_t n, int64_t texts, int heads) { return (texts ? n / texts : n) <= 64 || n / 128 * heads < 384 ? 64 : 128; }
// Texts of which the tiles far from a row are most: see walk().  (65,000 to 16,000 tokens, 16 heads of 64 bf16 values, without and with runs: 16 texts of 1,024 93.0 and 93.2 us (gradient 340,
// 320), 10 of 1,600 146 and 144 (531, 498), four of 4,096 319 and 304 (1,095, 1,041).)
inline bool long_texts(int64_t n, int64_t texts) { return texts > 0 && n / texts > 1024; }
// fp32 keeps to 64 rows but for long texts and the widest heads: a second workgroup a compute unit is worth more there than half of the reading.  (Forward, 8 heads, 64 and 128 rows: 200 texts
// of 200 tokens, heads of 64 values 278 and 374 us, 96 348 and 472, 128 609 and 595; four texts of 2,000, heads of 64 291 and 287.)
inline bool few_rows_of_floats(int64_t n, int64_t texts, int d) { return d <= 96 && !long_texts(n, texts); }

}  // namespace
}  // namespace pqt
