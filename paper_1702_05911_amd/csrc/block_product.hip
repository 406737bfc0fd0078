// Products of matrices in 8-bit blocks: out[i][j] = bias[j] + sum over k of A[i][k] B[j][k], where 128 consecutive k share a scale.
//
// bf16 results: the scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4 contracts one block of 128 at a time and multiplies by both
// scales itself (a byte exponent for every row and 32 values: the four of a block are the same), so that the sums stay in its
// accumulators from the first block to the last, in fp32.  B's rows are its first operand: a lane then holds four
// consecutive columns of the result.
//
// fp32 and f16 results: that instruction keeps of each product only what reaches 2^-13 of the largest of eight neighbouring products (measured,
// of the result's size: 1.4e-5 on normal data, 5.5e-5 where a few inputs are twenty times as large as the others; rounding to bf16 takes 1.7e-3, to
// f16 2.1e-4, so that f16 results came out up to 1.3 times as far off as their type makes them).  So the codes become bf16
// numbers under their scale, which loses nothing, and the bf16 instruction multiplies them, at half the rate; its sums are fp32 ones (9e-9).
//
// Three kernels, by the size of the result (plan_of):
//   wide   (bf16 results) 256 x 256 a workgroup of four wavefronts, one a SIMD, 128 x 128 each: half the bytes from LDS per multiplication of smaller ones
//   tile   128 x 128 or 64 x 64 a workgroup, two or four workgroups a compute unit; where there are few tiles, the blocks of k are shared
//          out over several workgroups, whose sums go to the workspace and are joined in order
//   few    up to 16 rows of A: B goes straight to registers, a wavefront has 16 of its rows, the wavefronts of a workgroup share out k
// The codes of a block of k go from memory straight to LDS (16 bytes a lane) while the blocks before are multiplied.  A row's eight 16-byte
// pieces lie there permuted by its number, so that the sixteen rows a fragment is read from fall into different banks (the lanes that a
// 16-byte LDS read serves together are 0-3, 12-15, 20-27 and so on: a lane takes pieces q and q + 4 of its row, q = lane / 16; which k those
// are is the same for both operands).  The two halves of what is double-buffered are LDS variables of their own: the compiler lets a
// read pass the loads that write another variable, and waits for all of them otherwise.
#include <algorithm>
#include <type_traits>

#include "encoder.hpp"
#include "product_plan.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const void global_bytes;
typedef __attribute__((address_space(3))) void lds_bytes;

constexpr int kBlock = PQT_BLOCK;
constexpr int64_t kMaxProduct = 0x0fffffff;    // rows of either side (of few rows of A: 512 threads for 64 of B's, fewer than 2^32 in all)
constexpr int64_t kMaxProductK = 1 << 22;      // (256 rows of codes are addressed by 32-bit offsets below 2^31)

struct ProductArgs {
    const uint8_t* a;
    const uint8_t* as;
    const uint8_t* b;
    const uint8_t* bs;
    const float* bias;
    void* out;
    float* parts;                          // splits x m x n, where the blocks of k are shared out
    int64_t out_stride;
    int m, n, kb;                          // kb: blocks of k
    int tiles_m, tiles_n;
    int splits, per_split;                 // blocks of k of a workgroup (even)
};

__device__ __forceinline__ f32x4 mfma_blocks(i32x8 b, i32x8 a, f32x4 c, uint32_t bs, uint32_t as) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, 0, (int)bs, 0, (int)as);
}

// the same with a block's codes as bf16: 2^(byte - 127) times each of a lane's 32
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
struct Wide { bf16x8 part[4]; };
__device__ __forceinline__ Wide widen(i32x8 codes, uint32_t byte) {
    const float scale = __uint_as_float((byte & 0xffu) << 23);
    Wide w;
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)codes[2 * p + h], scale, false);
            const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)codes[2 * p + h], scale, true);
            w.part[p][4 * h] = lo[0];
            w.part[p][4 * h + 1] = lo[1];
            w.part[p][4 * h + 2] = hi[0];
            w.part[p][4 * h + 3] = hi[1];
        }
    return w;
}
__device__ __forceinline__ f32x4 mfma_blocks(const Wide& b, const Wide& a, f32x4 c, uint32_t, uint32_t) {
#pragma unroll
    for (int p = 0; p < 4; ++p) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.part[p], a.part[p], c, 0, 0, 0);
    return c;
}
template <bool EXACT> struct Operand { typedef i32x8 type; };
template <> struct Operand<true> { typedef Wide type; };
template <bool EXACT>
__device__ __forceinline__ typename Operand<EXACT>::type operand(i32x8 codes, uint32_t byte) {
    if constexpr (EXACT) return widen(codes, byte);
    else return codes;
}

// Fragments of A's rows with one of B's.  bf16: a sum's four multiplications wait for each other, so the others come in between.
template <bool EXACT, int F>
__device__ __forceinline__ void multiply_row(f32x4 (&acc)[F], const typename Operand<EXACT>::type& b, const typename Operand<EXACT>::type (&a)[F],
                                             uint32_t sb, const uint32_t (&sa)[F]) {
    if constexpr (EXACT) {
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int j = 0; j < F; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.part[p], a[j].part[p], acc[j], 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < F; ++j) acc[j] = mfma_blocks(b, a[j], acc[j], sb, sa[j]);
    }
}

// vmcnt(N) lgkmcnt(0)
template <int N>
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x70); }

// Workgroup -> tile.  Consecutive workgroups go to the eight XCDs in turn: each gets a run of consecutive tiles, and these walk through eight
// rows of tiles column by column, so that what one XCD's L2 holds is used by its neighbours in time.
__device__ __forceinline__ void tile_of(const ProductArgs& g, int& tile_m, int& tile_n) {
    const int total = g.tiles_m * g.tiles_n, x = blockIdx.x & 7, j = blockIdx.x >> 3, per = total >> 3, more = total & 7;
    const int t = x * per + min(x, more) + j;
    constexpr int kRows = 8;
    const int of_group = kRows * g.tiles_n, group = t / of_group, first = group * kRows, rows = min(kRows, g.tiles_m - first), r = t - group * of_group;
    tile_m = first + r % rows;
    tile_n = r / rows;
}

// Rows row .. row + most of a matrix of codes, as a buffer: reading past them gives zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint8_t* codes, int row, int most, int rows, uint32_t kp) {
    const int have = min(max(rows - row, 0), most);
    const uint64_t at = (uint64_t)codes + (uint64_t)(have ? row : 0) * kp;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), (short)0, __builtin_amdgcn_readfirstlane((uint32_t)have * kp), 0x00027000);
}
constexpr uint32_t kNowhere = 0x80000000u;     // an offset past every buffer (256 rows of at most 2^22 bytes)

// Scale bytes of blocks k .. k + 7 of a row in one (unaligned) load; near the end of the array it begins earlier, and the shift puts it
// right.  Bytes past the row's end become zeros: what stands there for another row is not multiplied with this one's zeros.
struct EightScales {
    uint64_t bytes;
    uint32_t shift;
    int valid;
    __device__ __forceinline__ uint64_t value() const { return (bytes >> shift) & (~0ull >> (64 - 8 * valid)); }
};
__device__ __forceinline__ EightScales scales_of(const uint8_t* scales, int row, int rows, int k, int kb) {
    typedef uint64_t __attribute__((aligned(1))) bytes8;
    const int first = min(k, kb - 1), valid = min(8, kb - first);
    const int64_t total = (int64_t)rows * kb, want = (int64_t)min(row, rows - 1) * kb + first, at = min(want, total - 8);
    if (total < 8) {
        uint64_t v = 0;
        for (int i = 0; i < valid; ++i) v |= (uint64_t)scales[want + i] << (8 * i);
        return {v, 0, valid};
    }
    return {*reinterpret_cast<const bytes8*>(scales + at), (uint32_t)(want - at) * 8, valid};
}

// a lane's 32 bytes of row `row` of a tile in LDS: pieces q and q + 4
__device__ __forceinline__ i32x8 fragment(const uint8_t* tile, int row, int p0, int p1) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(tile + row * kBlock + p0), hi = *reinterpret_cast<const i32x4*>(tile + row * kBlock + p1);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <typename TY>
__device__ __forceinline__ void store_result(const ProductArgs& g, int row, int col, f32x4 v) {
    const int have = min(4, g.n - col);
    if (row >= g.m || have <= 0) return;
    if (g.splits > 1) {
        store_piece<float, 4>(g.parts + ((size_t)blockIdx.y * g.m + row) * g.n + col, v, have);
        return;
    }
    if (g.bias) v = v + load_piece<float, 4>(g.bias + col, have);
    store_piece<TY, 4>(static_cast<TY*>(g.out) + (int64_t)row * g.out_stride + col, v, have);
}

// ---- tile -----------------------------------------------------------------------------------------------------------
// Four wavefronts, each a quarter of the tile.  A block of k is multiplied while the next is on its way; with two to four workgroups a
// compute unit others multiply while this one waits.  fp32 and f16 results: half of the rate of the bf16 instructions (8192 x 8192 x 8192 1.2 PFLOP/s);
// the conversions, two a multiplication, hide beside them, the waits of a step do not.
template <typename TY, int B>
__global__ __launch_bounds__(256, B == 128 ? 2 : 4) void product_tile_kernel(ProductArgs g) {
    constexpr bool kExact = !std::is_same_v<TY, Bf16>;
    constexpr int F = B / 32, kLoads = B / 32;                  // fragments of a wavefront and loads of a lane, either side
    __shared__ __align__(16) uint8_t even[2 * B * kBlock];
    __shared__ __align__(16) uint8_t odd[2 * B * kBlock];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wm = wave / 2, wn = wave % 2, fr = lane & 15, q = lane >> 4;
    int tile_m, tile_n;
    tile_of(g, tile_m, tile_n);
    const int m0 = tile_m * B, n0 = tile_n * B;
    const int k0 = (int)blockIdx.y * g.per_split, k1 = min(g.kb, k0 + g.per_split);
    const uint32_t kp = (uint32_t)g.kb * kBlock;
    uint32_t off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = tid / 8 + i * 32;
        off[i] = (uint32_t)r * kp + ((tid & 7) ^ ((r >> 1) & 7)) * 16;
    }
    const __amdgpu_buffer_rsrc_t ra = rows_of(g.a, m0, B, g.m, kp), rb = rows_of(g.b, n0, B, g.n, kp);
    auto fetch = [&](uint8_t* tile, int k) __attribute__((always_inline)) {
        const bool in = k < k1;
        const int at = (in ? k : k0) * kBlock;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t o = in ? off[i] : kNowhere;          // past the last block: zeros
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_bytes*)(tile + (i * 32 + wave * 8) * kBlock), 16, o, at, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_bytes*)(tile + (B + i * 32 + wave * 8) * kBlock), 16, o, at, 0, 0);
        }
    };
    f32x4 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = 0.0f;
    // a lane holds the scales of one row of either side (B = 64: lanes 32 .. 63 those of lanes 0 .. 31 again), passed on when they are needed
    const int of_wave = B / 2;
    EightScales ha = scales_of(g.as, m0 + wm * of_wave + (lane & (of_wave - 1)), g.m, k0, g.kb), hb = scales_of(g.bs, n0 + wn * of_wave + (lane & (of_wave - 1)), g.n, k0, g.kb);
    uint64_t va = ha.value(), vb = hb.value();
    const int p0 = (q ^ ((fr >> 1) & 7)) * 16, p1 = ((q + 4) ^ ((fr >> 1) & 7)) * 16;
    const int row_a = wm * of_wave + fr, row_b = B + wn * of_wave + fr;
    uint32_t sa[F], sb[F];
    auto pass_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            sa[i] = (uint32_t)__builtin_amdgcn_ds_bpermute((i * 16 + fr) * 4, (int)va);
            sb[i] = (uint32_t)__builtin_amdgcn_ds_bpermute((i * 16 + fr) * 4, (int)vb);
        }
        va >>= 8;
        vb >>= 8;
    };
    typename Operand<kExact>::type fa[F], fb;
    // One block, whose fragments of A and first of B are there: while one of B is multiplied the next is read.  The last one's time
    // goes with the next block's, so the workgroup meets before that: the next block is there, and nobody reads this one any more.
    auto step = [&](int k, uint8_t* cur, const uint8_t* next) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i + 1 < F; ++i) {
            const i32x8 b = fragment(cur, row_b + (i + 1) * 16, p0, p1);
            multiply_row<kExact, F>(acc[i], fb, fa, sb[i], sa);
            fb = operand<kExact>(b, sb[i + 1]);
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        fetch(cur, k + 2);
        i32x8 a[F];
#pragma unroll
        for (int j = 0; j < F; ++j) a[j] = fragment(next, row_a + j * 16, p0, p1);
        const i32x8 b = fragment(next, row_b, p0, p1);
        multiply_row<kExact, F>(acc[F - 1], fb, fa, sb[F - 1], sa);
        pass_scales();
#pragma unroll
        for (int j = 0; j < F; ++j) fa[j] = operand<kExact>(a[j], sa[j]);
        fb = operand<kExact>(b, sb[0]);
    };
    fetch(even, k0);
    fetch(odd, k0 + 1);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    pass_scales();
#pragma unroll
    for (int j = 0; j < F; ++j) fa[j] = operand<kExact>(fragment(even, row_a + j * 16, p0, p1), sa[j]);
    fb = operand<kExact>(fragment(even, row_b, p0, p1), sb[0]);
    for (int k = k0; k < k1; k += 2) {
        if (((k - k0) & 7) == 4) {                              // two blocks before they are taken
            ha = scales_of(g.as, m0 + wm * of_wave + (lane & (of_wave - 1)), g.m, k + 4, g.kb);
            hb = scales_of(g.bs, n0 + wn * of_wave + (lane & (of_wave - 1)), g.n, k + 4, g.kb);
        }
        step(k, even, odd);
        if (((k - k0) & 7) == 6) {                              // (the block after the next begins eight new ones)
            va = ha.value();
            vb = hb.value();
        }
        step(k + 1, odd, even);
    }
    __builtin_amdgcn_s_waitcnt(0);                              // (what was fetched past the end)
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) store_result<TY>(g, m0 + wm * of_wave + j * 16 + fr, n0 + wn * of_wave + i * 16 + q * 4, acc[i][j]);
}

// ---- wide -----------------------------------------------------------------------------------------------------------
// A wavefront has a SIMD to itself, so what it waits for nobody covers.  Its instructions are laid out by hand: four
// multiplications, in their shadow one fragment read from LDS and one load to LDS, eight times a half block.  A half tile (lo: rows
// with bit 6 clear, hi: the others; A's 128, then B's) is free for the block after the next as soon as its last fragment is read:
//   first half   barrier; loads lo of k + 2; reads hi of k; multiplies A lo with B lo, then with B hi
//   second half  barrier; loads hi of k + 2; reads lo of k + 1; multiplies A hi with B lo, then with B hi
// so that a load has one and a half blocks of time, and 16 loads (of the two halves after it) may still be out when it is waited for.
// 8192 x 8192 x 8192 2.9 PFLOP/s, 16384 x 4096 x 4096 2.5 (216 us by itself, 220 behind the cutting of A, 263 at the median under a profiler); this card's instruction by itself
// 4.0 on such data (its clock falls), with wavefronts of 64 x 128, two a SIMD, whose fragments take all of LDS's rate, 1.9.  A block of k
// takes 1.26 us, the first loads and the result of a tile 14, in which nothing is multiplied: tiles in one long-lived workgroup with stores
// straight from the registers were slower (249), as their sums did not stay in registers.
__global__ __launch_bounds__(256, 1) void product_wide_kernel(ProductArgs g) {
    typedef Bf16 TY;
    constexpr int B = 256, F = 8, kHalf = B * kBlock;
    __shared__ __align__(16) uint8_t lo_even[kHalf];
    __shared__ __align__(16) uint8_t hi_even[kHalf];
    __shared__ __align__(16) uint8_t lo_odd[kHalf];
    __shared__ __align__(16) uint8_t hi_odd[kHalf];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wm = wave / 2, wn = wave % 2, fr = lane & 15, q = lane >> 4;
    int tile_m, tile_n;
    tile_of(g, tile_m, tile_n);
    const int m0 = tile_m * B, n0 = tile_n * B;
    const uint32_t kp = (uint32_t)g.kb * kBlock;
    uint32_t off[4];                                            // place p of a half tile's side: row (p & 63) + 2 (p & 64)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int p = tid / 8 + i * 32;
        off[i] = (uint32_t)((p & 63) + 2 * (p & 64)) * kp + ((tid & 7) ^ ((p >> 1) & 7)) * 16;
    }
    const __amdgpu_buffer_rsrc_t a_lo = rows_of(g.a, m0, B, g.m, kp), a_hi = rows_of(g.a, m0 + 64, B, g.m, kp);
    const __amdgpu_buffer_rsrc_t b_lo = rows_of(g.b, n0, B, g.n, kp), b_hi = rows_of(g.b, n0 + 64, B, g.n, kp);
    // one of the eight loads of a half tile
    auto fetch = [&](uint8_t* half, const __amdgpu_buffer_rsrc_t& ra, const __amdgpu_buffer_rsrc_t& rb, int k, int e) __attribute__((always_inline)) {
        const bool in = k < g.kb;
        const int at = (in ? k : 0) * kBlock, i = e >> 1;
        const uint32_t o = in ? off[i] : kNowhere;              // past the last block: zeros
        if (e & 1) __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_bytes*)(half + (128 + i * 32 + wave * 8) * kBlock), 16, o, at, 0, 0);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_bytes*)(half + (i * 32 + wave * 8) * kBlock), 16, o, at, 0, 0);
    };
    // a lane holds the scales of two rows of either side, eight blocks' at a time, and passes on the bytes of two blocks
    EightScales held[4];
    uint64_t bytes[4];
    uint32_t sa[F], sb[F];
    auto fetch_scales = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            held[i] = scales_of(g.as, m0 + wm * 128 + i * 64 + lane, g.m, k, g.kb);
            held[2 + i] = scales_of(g.bs, n0 + wn * 128 + i * 64 + lane, g.n, k, g.kb);
        }
    };
    auto take_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) bytes[i] = held[i].value();
    };
    auto pass_scales = [&](int shift) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < F; ++j) {
            sa[j] = (uint32_t)__builtin_amdgcn_ds_bpermute(((j & 3) * 16 + fr) * 4, (int)(bytes[j >> 2] >> shift));
            sb[j] = (uint32_t)__builtin_amdgcn_ds_bpermute(((j & 3) * 16 + fr) * 4, (int)(bytes[2 + (j >> 2)] >> shift));
        }
    };
    f32x4 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = 0.0f;
    const int p0 = (q ^ ((fr >> 1) & 7)) * 16, p1 = ((q + 4) ^ ((fr >> 1) & 7)) * 16;
    const int row_a = wm * 64 + fr, row_b = 128 + wn * 64 + fr;
    i32x8 a0[4], a1[4], b0[4], b1[4];                           // fragments of A lo, A hi, B lo, B hi
    auto four = [&](const i32x8 (&a)[4], const i32x8& b, int ha, int ib) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[ib][ha * 4 + j] = mfma_blocks(b, a[j], acc[ib][ha * 4 + j], sb[ib], sa[ha * 4 + j]);
    };
    // the order of what one group of four multiplications goes with: reads, a load, and the multiplications between them
    auto lay_out = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto meet = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<16>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    // one block of k, whose A lo and B lo fragments are there
    auto step = [&](int k, auto is_odd, uint8_t* lo, uint8_t* hi, uint8_t* lo_next) __attribute__((always_inline)) {
        meet();
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (u < 2) {
                b1[2 * u] = fragment(hi, row_b + 2 * u * 16, p0, p1);
                b1[2 * u + 1] = fragment(hi, row_b + (2 * u + 1) * 16, p0, p1);
            } else if (u < 6) a1[u - 2] = fragment(hi, row_a + (u - 2) * 16, p0, p1);
            fetch(lo, a_lo, b_lo, k + 2, u);
            if (u < 4) four(a0, b0[u], 0, u); else four(a0, b1[u - 4], 0, u);
            lay_out();
        }
        meet();
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (u < 4) a0[u] = fragment(lo_next, row_a + u * 16, p0, p1);
            else if (u < 6) {                                   // (B lo's are free now)
                b0[2 * (u - 4)] = fragment(lo_next, row_b + 2 * (u - 4) * 16, p0, p1);
                b0[2 * (u - 4) + 1] = fragment(lo_next, row_b + (2 * (u - 4) + 1) * 16, p0, p1);
            }
            fetch(hi, a_hi, b_hi, k + 2, u);
            if (u < 4) four(a1, b0[u], 1, u); else four(a1, b1[u - 4], 1, u);
            lay_out();
        }
        if (is_odd.value) pass_scales(((k + 1) & 7) * 8);
        else {
#pragma unroll
            for (int j = 0; j < F; ++j) {
                sa[j] >>= 8;
                sb[j] >>= 8;
            }
        }
    };
    fetch_scales(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) fetch(lo_even, a_lo, b_lo, 0, e);
    __builtin_amdgcn_sched_barrier(0);                          // (loads are waited for by their number: the halves stay in order)
#pragma unroll
    for (int e = 0; e < 8; ++e) fetch(hi_even, a_hi, b_hi, 0, e);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) fetch(lo_odd, a_lo, b_lo, 1, e);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) fetch(hi_odd, a_hi, b_hi, 1, e);
    __builtin_amdgcn_sched_barrier(0);
    wait_loads<24>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    take_scales();
    pass_scales(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) a0[i] = fragment(lo_even, row_a + i * 16, p0, p1);
#pragma unroll
    for (int i = 0; i < 4; ++i) b0[i] = fragment(lo_even, row_b + i * 16, p0, p1);
    for (int k = 0; k < g.kb; k += 2) {
        if ((k & 7) == 4) fetch_scales(k + 4);                  // two blocks before they are taken, four before they are used
        if ((k & 7) == 6) take_scales();
        step(k, std::integral_constant<bool, false>{}, lo_even, hi_even, lo_odd);
        step(k + 1, std::integral_constant<bool, true>{}, lo_odd, hi_odd, lo_even);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // The tile as TY through LDS, 64 rows in each half tile's room (pieces permuted by the row again), so that rows are written as a whole.
    typedef typename Piece_<TY, 4>::type V4;
    uint8_t* lower = wm ? lo_odd : lo_even;
    uint8_t* upper = wm ? hi_odd : hi_even;
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const int col = wn * 128 + i * 16 + q * 4;
        f32x4 bias = {0.0f, 0.0f, 0.0f, 0.0f};
        if (g.bias) {
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[e] = g.bias[min(n0 + col + e, g.n - 1)];
        }
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int at = ((j & 3) * 16 + fr) * (2 * B) + (((col >> 3) ^ fr) << 4) + (q & 1) * 8;
            *reinterpret_cast<V4*>((j < 4 ? lower : upper) + at) = __builtin_convertvector(acc[i][j] + bias, V4);
        }
    }
    __syncthreads();
    const bool stream = (double)g.m * g.n * sizeof(TY) > kStreamBytes;
    const int unit = tid & 31, have = min(8, g.n - n0 - unit * 8);
    if (have <= 0) return;
#pragma unroll 1
    for (int h = 0; h < 4; ++h) {
        const uint8_t* half = h == 0 ? lo_even : h == 1 ? hi_even : h == 2 ? lo_odd : hi_odd;
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int r = p * 8 + (tid >> 5), row = m0 + h * 64 + r;
            if (row < g.m) {
                const TY* from = reinterpret_cast<const TY*>(half + r * (2 * B) + ((unit ^ (r & 15)) << 4));
                TY* dst = static_cast<TY*>(g.out) + (int64_t)row * g.out_stride + n0 + unit * 8;
                if (have == 8) store_vector(reinterpret_cast<typename Piece_<TY, 8>::type*>(dst), *reinterpret_cast<const typename Piece_<TY, 8>::type*>(from), stream);
                else
                    for (int e = 0; e < have; ++e) dst[e] = from[e];
            }
        }
    }
}

// the splits' sums, in order
template <typename TY>
__global__ __launch_bounds__(256) void join_splits_kernel(ProductArgs g) {
    const int pieces = (g.n + 3) / 4;
    const int64_t total = (int64_t)g.m * pieces;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
        const int row = (int)(e / pieces), col = (int)(e - (int64_t)row * pieces) * 4, have = min(4, g.n - col);
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < g.splits; ++s) v = v + load_piece<float, 4>(g.parts + ((size_t)s * g.m + row) * g.n + col, have);
        if (g.bias) v = v + load_piece<float, 4>(g.bias + col, have);
        store_piece<TY, 4>(static_cast<TY*>(g.out) + (int64_t)row * g.out_stride + col, v, have);
    }
}

// ---- few rows of A --------------------------------------------------------------------------------------------------
constexpr int kFewWaves = 8, kFewRun = 4;

// A wavefront multiplies 16 NF rows of B with all of A's over every kFewWaves-th run of four blocks, all of whose loads are sent first; the sums
// of the wavefronts are added in order.  Bound by the reading of B: 1 x 4096 x 4096 4.8 us with B in the caches, 6.2 from memory (2.7 TB/s: one
// round of loads, whose latency it is); 16 x 32768 x 4096 24.6 from the caches, 5.5 TB/s (NF = 1: 35.1), 37 from memory.  bf16 results by the
// instructions of the others: 6.4, 38, and 4 x 40000 x 1000 16.7 for 14.5.
template <typename TY, int NF>
__global__ __launch_bounds__(kFewWaves * kWave) void product_few_kernel(ProductArgs g) {
    constexpr bool kExact = !std::is_same_v<TY, Bf16>;
    __shared__ f32x4 sums[kFewWaves][NF][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), fr = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * (16 * NF);
    const uint32_t kp = (uint32_t)g.kb * kBlock;
    const __amdgpu_buffer_rsrc_t ra = rows_of(g.a, 0, kFewRows, g.m, kp), rb = rows_of(g.b, n0, 16 * NF, g.n, kp);
    const uint32_t off = (uint32_t)fr * kp + q * 16;
    f32x4 acc[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[f] = 0.0f;
    for (int k = wave * kFewRun; k < g.kb; k += kFewWaves * kFewRun) {
        i32x4 a[kFewRun][2], b[NF][kFewRun][2];
        uint64_t sb[NF];
#pragma unroll
        for (int u = 0; u < kFewRun; ++u) {
            const uint32_t at = k + u < g.kb ? off + (uint32_t)(k + u) * kBlock : kNowhere;        // past the last block: zeros
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int h = 0; h < 2; ++h) b[f][u][h] = __builtin_amdgcn_raw_buffer_load_b128(rb, at + (uint32_t)(f * 16) * kp, h * 64, 0);
#pragma unroll
            for (int h = 0; h < 2; ++h) a[u][h] = __builtin_amdgcn_raw_buffer_load_b128(ra, at, h * 64, 0);
        }
        const uint64_t sa = scales_of(g.as, fr, g.m, k, g.kb).value();
#pragma unroll
        for (int f = 0; f < NF; ++f) sb[f] = scales_of(g.bs, n0 + f * 16 + fr, g.n, k, g.kb).value();
#pragma unroll
        for (int u = 0; u < kFewRun; ++u) {
            const uint32_t va = (uint32_t)(sa >> (8 * u));
            const auto oa = operand<kExact>(__builtin_shufflevector(a[u][0], a[u][1], 0, 1, 2, 3, 4, 5, 6, 7), va);
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const uint32_t vb = (uint32_t)(sb[f] >> (8 * u));
                acc[f] = mfma_blocks(operand<kExact>(__builtin_shufflevector(b[f][u][0], b[f][u][1], 0, 1, 2, 3, 4, 5, 6, 7), vb), oa, acc[f], vb, va);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) sums[wave][f][lane] = acc[f];
    __syncthreads();
    if (wave >= NF) return;
    f32x4 v = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) v = v + sums[w][wave][lane];
    store_result<TY>(g, fr, n0 + wave * 16 + q * 4, v);
}

}  // namespace
}  // namespace pqt

extern "C" {

size_t pqt_block_product_workspace(int64_t m, int64_t n, int64_t k) {
    if (m < 1 || n < 1 || k < 1 || m > pqt::kMaxProduct || n > pqt::kMaxProduct || k > pqt::kMaxProductK) return 0;
    const int kb = (int)((k + pqt::kBlock - 1) / pqt::kBlock);
    const int splits = std::max(pqt::plan_of(m, n, kb, false).splits, pqt::plan_of(m, n, kb, true).splits);
    return splits > 1 ? sizeof(float) * (size_t)splits * (size_t)m * (size_t)n : 0;
}

int pqt_block_product(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales, int64_t m,
                      int64_t n, int64_t k, const float* bias, void* out, int out_type, int64_t out_stride, void* workspace,
                      size_t workspace_bytes, int device, void* hip_stream) {
    using namespace pqt;
    if (!known_type(out_type)) return fail(PQT_EINVAL, "pqt_block_product: unknown type %d", out_type);
    if (m < 0 || n < 0 || k < 1 || out_stride < n)
        return fail(PQT_EINVAL, "pqt_block_product: m=%lld n=%lld k=%lld stride=%lld out of range", (long long)m, (long long)n, (long long)k, (long long)out_stride);
    if (m > kMaxProduct || n > kMaxProduct || k > kMaxProductK)
        return fail(PQT_EUNSUPPORTED, "pqt_block_product: m=%lld n=%lld k=%lld beyond the limits", (long long)m, (long long)n, (long long)k);
    if (m == 0 || n == 0) return PQT_OK;
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return fail(PQT_EINVAL, "pqt_block_product: null pointer");
    if (!aligned_to(a_codes, 16) || !aligned_to(b_codes, 16) || !aligned_to(out, type_bytes(out_type)) || !aligned_to(bias, 4))
        return fail(PQT_EINVAL, "pqt_block_product: a pointer is not aligned (codes to 16 bytes, the others to their element)");
    const size_t need = pqt_block_product_workspace(m, n, k);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_block_product: workspace of %zu bytes, aligned to 16, needed (%zu given)", need, workspace_bytes);
    const int kb = (int)((k + kBlock - 1) / kBlock);
    const Plan p = plan_of(m, n, kb, out_type != PQT_BF16);
    if ((int64_t)p.tiles_m * p.tiles_n > kMaxTiles)
        return fail(PQT_EUNSUPPORTED, "pqt_block_product: %d x %d tiles", p.tiles_m, p.tiles_n);
    if (const int rc = check_device(device, "pqt_block_product")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const ProductArgs g{a_codes, a_scales, b_codes, b_scales, bias, out, static_cast<float*>(workspace), out_stride, (int)m, (int)n, kb,
                        p.tiles_m, p.tiles_n, p.splits, p.per_split};
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n), (unsigned)p.splits);
    with_type(out_type, [&](auto y) {
        using TY = decltype(y);
        if (p.tile == 16 && n >= kManyColumns) hipLaunchKernelGGL((product_few_kernel<TY, 4>), dim3((unsigned)((n + 63) / 64)), dim3(kFewWaves * kWave), 0, st, g);
        else if (p.tile == 16) hipLaunchKernelGGL((product_few_kernel<TY, 1>), dim3((unsigned)((n + 15) / 16)), dim3(kFewWaves * kWave), 0, st, g);
        else if (p.tile == 64) hipLaunchKernelGGL((product_tile_kernel<TY, 64>), grid, dim3(256), 0, st, g);
        else if (p.tile == 128) hipLaunchKernelGGL((product_tile_kernel<TY, 128>), grid, dim3(256), 0, st, g);
        else if constexpr (std::is_same_v<TY, Bf16>) hipLaunchKernelGGL(product_wide_kernel, grid, dim3(256), 0, st, g);
    });
    HIP_TRY(hipGetLastError());
    if (p.splits > 1) {
        const int64_t work = (m * ((n + 3) / 4) + 255) / 256;
        with_type(out_type, [&](auto y) {
            hipLaunchKernelGGL((join_splits_kernel<decltype(y)>), dim3((unsigned)std::min<int64_t>(work, 4096)), dim3(256), 0, st, g);
        });
        HIP_TRY(hipGetLastError());
    }
    return PQT_OK;
}

}  // extern "C"
