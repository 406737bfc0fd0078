// A matrix cut into 8-bit blocks: 128 values of a row (or of a column, for the transpose) share a power of two that brings the largest
// of them to at most 448, the largest e4m3 number, and are rounded to the nearest e4m3 number.
//
// Bound by memory: two or four bytes a value read, one written for each of the two forms.  Rows alone: sixteen lanes hold a block, eight
// values each, and find its largest value among themselves; nothing goes through LDS.  With columns: a workgroup of 512 threads
// holds a tile of 128 x 128, a thread four rows of eight columns, so that both forms' maxima are found in registers and
// over few lanes, and the transposed bytes of four rows make one 4-byte piece; those go through LDS, from where they
// are written as whole blocks of 128 bytes.
// Measured: rows alone 16,384 x 4,096 bf16 41 us, 4.9 TB/s (a large copy 5.1); both forms 8,191 x 2,000 20 us, 3.2 TB/s (27.6 by 256
// threads of eight rows each, whose loads stood behind conditions: too few on their way).
#include <algorithm>

#include "block_codes.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

constexpr int kQuantThreads = 256;

struct QuantizeArgs {
    const void* x;
    int64_t rows, cols, x_stride;
    uint8_t* codes;
    uint8_t* scales;
    uint8_t* codes_t;
    uint8_t* scales_t;
};

// Eight values of a row from column c on, zeros past its end.  The load is unconditional, so that several of a thread's are on their way at once:
// a piece that is not whole is read from an earlier column first, and again by the lanes that have one.
template <typename T>
__device__ __forceinline__ typename Piece_<T, 8>::type eight_of(const T* row, int64_t c, int64_t cols) {
    return cols >= 8 ? WholePiece<8>(c, cols).template load<T>(row) : typename Piece_<T, 8>::type{};
}
template <typename T>
__device__ __forceinline__ typename Piece_<T, 8>::type put_right(typename Piece_<T, 8>::type v, const T* row, int64_t c, int64_t cols) {
    if (c + 8 > cols) v = load_raw<T, 8>(row + (c < cols ? c : 0), (int)max(cols - c, (int64_t)0));
    return v;
}

// blocks along rows, one by sixteen lanes
constexpr int64_t kRowsGrid = 1 << 20;

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(QuantizeArgs g, int blocks_of_row) {
    const int64_t total = g.rows * blocks_of_row;
    const int l = threadIdx.x & (kLanesOfBlock - 1);
    const int64_t step = (int64_t)gridDim.x * (kQuantThreads / kLanesOfBlock);
    for (int64_t i = (int64_t)blockIdx.x * (kQuantThreads / kLanesOfBlock) + threadIdx.x / kLanesOfBlock; i < total; i += step) {
        const int64_t r = total <= 0xffffffff ? (int64_t)((uint32_t)i / (uint32_t)blocks_of_row) : i / blocks_of_row;
        const int64_t c = (i - r * blocks_of_row) * kBlock + l * 8;
        const T* row = static_cast<const T*>(g.x) + r * g.x_stride;
        const f32x8 v = __builtin_convertvector(put_right(eight_of(row, c, g.cols), row, c, g.cols), f32x8);
        float e[8];
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = v[j];
            m = max(m, magnitude(e[j]));
        }
        const bool all_finite = __ballot(m >= kNotFinite) == 0;
        if (!all_finite) {
            m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, finite_magnitude(e[j]));
        }
        const uint32_t byte = scale_byte(max_of_16(m));
        *reinterpret_cast<uint2*>(g.codes + (i * kBlock + l * 8)) = eight_codes(e, inverse_scale(byte), all_finite);
        if (l == 0) g.scales[i] = (uint8_t)byte;
    }
}

// A tile of 128 x 128, blocks down its columns and, where codes is not null, along its rows.  A thread has four rows of eight columns.
constexpr int kTileThreads = 512, kTileRows = 4;

template <typename T>
__global__ __launch_bounds__(kTileThreads) void quantize_tile_kernel(QuantizeArgs g, int blocks_of_row, int blocks_of_col) {
    constexpr int kPitch = kBlock + 4;                         // (of a column's bytes: eight columns apart is eight banks apart)
    constexpr int kWaves = kTileThreads / kWave;
    __shared__ __align__(16) uint8_t turned[kBlock * kPitch];
    __shared__ uint32_t maxima[kWaves][kBlock];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int pc = tid & 15, pr = tid >> 4;
    const int bc = (int)(blockIdx.x % (unsigned)blocks_of_row);
    const int64_t br = blockIdx.x / (unsigned)blocks_of_row;
    const int64_t r0 = br * kBlock + pr * kTileRows, c0 = (int64_t)bc * kBlock + pc * 8;
    typename Piece_<T, 8>::type raw[kTileRows];
    const T* x = static_cast<const T*>(g.x);
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) raw[i] = eight_of(x + min(r0 + i, g.rows - 1) * g.x_stride, c0, g.cols);
    float v[kTileRows][8];
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < kTileRows; ++i) {
        raw[i] = put_right(raw[i], x + min(r0 + i, g.rows - 1) * g.x_stride, c0, g.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[i][j] = r0 + i < g.rows ? (float)raw[i][j] : 0.0f;
            all = max(all, magnitude(v[i][j]));
        }
    }
    const bool all_finite = __ballot(all >= kNotFinite) == 0;
    if (g.codes) {
#pragma unroll
        for (int i = 0; i < kTileRows; ++i) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, all_finite ? magnitude(v[i][j]) : finite_magnitude(v[i][j]));
            const uint32_t byte = scale_byte(max_of_16(m));
            if (r0 + i < g.rows) {
                const int64_t at = (r0 + i) * blocks_of_row + bc;
                *reinterpret_cast<uint2*>(g.codes + at * kBlock + pc * 8) = eight_codes(v[i], inverse_scale(byte), all_finite);
                if (pc == 0) g.scales[at] = (uint8_t)byte;
            }
        }
    }
    uint32_t top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kTileRows; ++i) m = max(m, all_finite ? magnitude(v[i][j]) : finite_magnitude(v[i][j]));
        m = max(m, (uint32_t)__builtin_amdgcn_ds_swizzle((int)m, (16 << 10) | 0x1f));
        top[j] = max(m, (uint32_t)__shfl_xor((int)m, 32, kWave));
    }
    if (lane < 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) maxima[wave][pc * 8 + j] = top[j];
    }
    __syncthreads();
    if (tid < kBlock) {                                        // the columns' scales, in the first wavefront's row
        uint32_t m = maxima[0][tid];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = max(m, maxima[w][tid]);
        const uint32_t byte = scale_byte(m);
        maxima[0][tid] = byte;
        const int64_t c = (int64_t)bc * kBlock + tid;
        if (c < g.cols) g.scales_t[c * blocks_of_col + br] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; j += 2) {                           // two columns' four rows
        float e[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float inv = inverse_scale(maxima[0][pc * 8 + j + h]);
#pragma unroll
            for (int i = 0; i < kTileRows; ++i) e[h * kTileRows + i] = magnitude(v[i][j + h]) >= kNotFinite ? v[i][j + h] : v[i][j + h] * inv;
        }
        const uint2 out = eight_codes(e, 1.0f, all_finite);
        *reinterpret_cast<uint32_t*>(turned + (pc * 8 + j) * kPitch + pr * kTileRows) = out.x;
        *reinterpret_cast<uint32_t*>(turned + (pc * 8 + j + 1) * kPitch + pr * kTileRows) = out.y;
    }
    __syncthreads();
    for (int e = tid; e < kBlock * (kBlock / 8); e += kTileThreads) {           // 8 bytes of a column
        const int col = e / (kBlock / 8), part = e & (kBlock / 8 - 1);
        const int64_t c = (int64_t)bc * kBlock + col;
        const uint32_t* from = reinterpret_cast<const uint32_t*>(turned + col * kPitch + part * 8);
        if (c < g.cols) *reinterpret_cast<uint2*>(g.codes_t + (c * blocks_of_col + br) * kBlock + part * 8) = uint2{from[0], from[1]};
    }
}

}  // namespace
}  // namespace pqt

extern "C" int pqt_block_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t x_stride, uint8_t* codes, uint8_t* scales,
                                  uint8_t* codes_t, uint8_t* scales_t, int device, void* hip_stream) {
    using namespace pqt;
    if (!known_type(type)) return fail(PQT_EINVAL, "pqt_block_quantize: unknown type %d", type);
    if (rows < 0 || cols < 1 || x_stride < cols)
        return fail(PQT_EINVAL, "pqt_block_quantize: rows=%lld cols=%lld stride=%lld out of range", (long long)rows, (long long)cols, (long long)x_stride);
    if (rows > 0x7fffffff || cols > 0x7fffff00) return fail(PQT_EUNSUPPORTED, "pqt_block_quantize: rows=%lld cols=%lld beyond 2^31", (long long)rows, (long long)cols);
    if (rows == 0) return PQT_OK;
    if (!x || !codes != !scales || !codes_t != !scales_t || (!codes && !codes_t)) return fail(PQT_EINVAL, "pqt_block_quantize: null pointer");
    if (!aligned_to(x, type_bytes(type)) || !aligned_to(codes, 16) || !aligned_to(codes_t, 16))
        return fail(PQT_EINVAL, "pqt_block_quantize: a pointer is not aligned (x to its element, codes to 16 bytes)");
    const int64_t of_row = (cols + kBlock - 1) / kBlock, of_col = (rows + kBlock - 1) / kBlock;
    if (codes_t && of_row * of_col > 0x7fffff) return fail(PQT_EUNSUPPORTED, "pqt_block_quantize: a transpose of %lld x %lld blocks", (long long)of_col, (long long)of_row);
    if (const int rc = check_device(device, "pqt_block_quantize")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const QuantizeArgs g{x, rows, cols, x_stride, codes, scales, codes_t, scales_t};
    with_type(type, [&](auto t) {
        if (codes_t) {
            hipLaunchKernelGGL((quantize_tile_kernel<decltype(t)>), dim3((unsigned)(of_row * of_col)), dim3(kTileThreads), 0, st, g, (int)of_row, (int)of_col);
        } else {
            const int64_t blocks = (rows * of_row + kQuantThreads / kLanesOfBlock - 1) / (kQuantThreads / kLanesOfBlock);
            hipLaunchKernelGGL((quantize_rows_kernel<decltype(t)>), dim3((unsigned)std::min<int64_t>(blocks, kRowsGrid)), dim3(kQuantThreads), 0, st, g, (int)of_row);
        }
    });
    HIP_TRY(hipGetLastError());
    return PQT_OK;
}
