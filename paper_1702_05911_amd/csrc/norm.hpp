// What layer norm and root-mean-square norm share (layer_norm.hip, rms_norm.hip): rows by groups of lanes, parameters, sums over a row, and
// the columns' sums of the gradients.
#pragma once
#include <algorithm>

#include "encoder.hpp"

namespace pqt {
namespace {

constexpr int kNormE = 8;                  // values of a piece
constexpr int64_t kMaxNormD = 32768;       // 1,024 lanes, four pieces
constexpr int kGradThreads = 512;
// The longest rows that the one-pass backward kernel takes: 8,192 floats (4,000 rows of 8,200: 187 us a call by it, 154 by two
// kernels), twice as many 16-bit values, which wait in half the registers (2,000 x 16,384 73 us, by two kernels 104)
inline int64_t one_pass_values(int type) { return type == PQT_F32 ? 8192 : 16384; }
constexpr unsigned kLongParts = 64;        // parts of the rows whose columns are added up one after the other beyond that
constexpr unsigned kGradBlocks = 256;      // workgroups of the backward pass, at most: one a compute unit

// eight values of a parameter (of any type), or `fill` where there is none
__device__ __forceinline__ f32x8 param_piece(const void* p, int type, int c, int have, float fill) {
    if (!p) {
        f32x8 v;
        v = fill;
        return v;
    }
    if (type == PQT_F32) return load_piece<float, kNormE>(static_cast<const float*>(p) + c, have);
    if (type == PQT_BF16) return load_piece<Bf16, kNormE>(static_cast<const Bf16*>(p) + c, have);
    return load_piece<Half, kNormE>(static_cast<const Half*>(p) + c, have);
}

// Zeros past a row's end, whatever stands there: (0 - mean) * rstd may leave fp32, and its product with a gradient of zero is NaN then.
__device__ __forceinline__ f32x8 up_to(f32x8 v, int have) {
    if (have < kNormE) {
        asm("" : "+v"(have));                  // (eight comparisons here, not their results kept in scalar registers over all rows)
#pragma unroll
        for (int j = 0; j < kNormE; ++j) v[j] = j < have ? v[j] : 0.0f;
    }
    return v;
}

__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// Sum over a group of G lanes; G > 64: over G / 64 wavefronts of a workgroup of whole groups, all of which call it (scratch: one value a
// wavefront, twice, used in turn, so that one barrier a sum is enough).
template <int G>
__device__ __forceinline__ float row_sum(float v, float (*scratch)[16], int& turn) {
    v = group_sum<(G < kWave ? G : kWave)>(v);
    if constexpr (G > kWave) {
        const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
        constexpr int W = G / kWave;
        if (lane == 0) scratch[turn][wave] = v;
        __syncthreads();
        const int w0 = wave & ~(W - 1);
        v = scratch[turn][w0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += scratch[turn][w0 + w];
        turn ^= 1;
    }
    return v;
}

// Sums of `columns` columns of the workgroups' rows, 64 a workgroup, its sixteen wavefronts a part of the rows each: the first D are dweight, what
// follows is dbias
__global__ __launch_bounds__(1024) void columns_kernel(const float* parts, int rows, int columns, int D, float* dweight, float* dbias) {
    __shared__ float sums[16][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int c = blockIdx.x * kWave + lane;
    float s = 0.0f;
    if (c < columns) {
        for (int r = wave; r < rows; r += 16 * 8) {            // eight rows on their way
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = parts[(size_t)min(r + 16 * u, rows - 1) * columns + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += r + 16 * u < rows ? v[u] : 0.0f;
        }
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= columns) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    float* out = c < D ? dweight : dbias;
    if (out) out[c < D ? c : c - D] = s;
}

// Calls f(G, NP): lanes of a group and pieces of a lane for rows of D values.  Up to 2,048 values a wavefront has a row by itself, up to four
// pieces a lane; then 256 threads, then 1,024.
template <int V> struct Int { static constexpr int value = V; };
template <typename F>
void with_shape(int64_t D, F&& f) {
    const int64_t pieces = (D + kNormE - 1) / kNormE;
    if (pieces <= 8) f(Int<8>{}, Int<1>{});
    else if (pieces <= 16) f(Int<16>{}, Int<1>{});
    else if (pieces <= 32) f(Int<32>{}, Int<1>{});
    else if (pieces <= 64) f(Int<64>{}, Int<1>{});
    else if (pieces <= 128) f(Int<64>{}, Int<2>{});
    else if (pieces <= 256) f(Int<64>{}, Int<4>{});
    else if (pieces <= 512) f(Int<256>{}, Int<2>{});
    else if (pieces <= 1024) f(Int<256>{}, Int<4>{});
    else if (pieces <= 2048) f(Int<1024>{}, Int<2>{});
    else f(Int<1024>{}, Int<4>{});
}
// The same for the backward pass, which holds five values for each of a row's: two pieces a lane at most.
template <typename F>
void with_gradient_shape(int64_t D, F&& f) {
    const int64_t pieces = (D + kNormE - 1) / kNormE;
    if (pieces <= 8) f(Int<8>{}, Int<1>{});
    else if (pieces <= 16) f(Int<16>{}, Int<1>{});
    else if (pieces <= 32) f(Int<32>{}, Int<1>{});
    else if (pieces <= 64) f(Int<64>{}, Int<1>{});
    else if (pieces <= 128) f(Int<64>{}, Int<2>{});
    else if (pieces <= 256) f(Int<128>{}, Int<2>{});
    else if (pieces <= 512) f(Int<256>{}, Int<2>{});
    else if (pieces <= 1024) f(Int<512>{}, Int<2>{});
    else f(Int<512>{}, Int<4>{});
}

// Workgroups of the backward kernel.  A single one for up to two rows a group: its sums are the result, without a second launch (8 x 1,000 bf16
// 4.6 us in a graph, by two launches 6.3.  Four rows a group: 32 x 1,000 7.9 and 6.8, 4 x 16,384 18.3 and 11.3).
constexpr int kAloneRows = 2;
unsigned gradient_blocks(int64_t rows, int groups) {
    return rows <= (int64_t)kAloneRows * groups ? 1u : (unsigned)std::min<int64_t>((rows + groups - 1) / groups, kGradBlocks);
}
unsigned gradient_blocks(int64_t rows, int64_t D, int type) {
    unsigned n = 0;
    if (D > one_pass_values(type)) return (unsigned)std::min<int64_t>(rows, kLongParts);
    with_gradient_shape(D, [&](auto G, auto) { n = gradient_blocks(rows, kGradThreads / G.value); });
    return n;
}

}  // namespace
}  // namespace pqt
