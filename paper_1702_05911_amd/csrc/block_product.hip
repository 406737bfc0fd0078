// Products of matrices in 8-bit blocks: out[i][j] = bias[j] + sum over k of A[i][k] B[j][k], where 128 consecutive k share a scale.
//
// Results of 16 bits: the scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4 contracts one block of 128 at a time and multiplies by both
// scales itself (a byte exponent for every row and 32 values: the four of a block are the same), so that the sums stay in its
// accumulators from the first block to the last, in fp32.  B's rows are its first operand: a lane then holds four
// consecutive columns of the result.
//
// tile kernel: a workgroup computes BM x BN.  The codes of a block of k go from memory straight to LDS, 16 bytes a lane, while the
// block before is multiplied; a row's eight 16-byte pieces lie there permuted by its number, so that the sixteen rows a
// fragment is read from fall into different banks.  Scales: four blocks' bytes a row in one register, shifted from block to block.
#include <algorithm>

#include "encoder.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const void global_bytes;
typedef __attribute__((address_space(3))) void lds_bytes;

constexpr int kBlock = PQT_BLOCK;

struct ProductArgs {
    const uint8_t* a;
    const uint8_t* as;
    const uint8_t* b;
    const uint8_t* bs;
    const float* bias;
    void* out;
    int64_t out_stride;
    int m, n, kb;                          // kb: blocks of k
    int tiles_m, tiles_n;
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

// the scale bytes of up to four blocks of a row, from block k on
__device__ __forceinline__ uint32_t scales_of(const uint8_t* row, int k, int kb) {
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (k + j < kb) v |= (uint32_t)row[k + j] << (8 * j);
    return v;
}

template <typename TY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void product_tile_kernel(ProductArgs g) {
    constexpr bool kExact = sizeof(TY) == 4;
    constexpr int T = 64 * WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kRowsA = BM / (T / 8), kRowsB = BN / (T / 8);        // 16-byte loads a thread
    __shared__ __align__(16) uint8_t codes[2][(BM + BN) * kBlock];
    __shared__ uint32_t scales[2][BM + BN];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wm = wave / WN, wn = wave % WN;
    const int tile_m = blockIdx.x % g.tiles_m, tile_n = blockIdx.x / g.tiles_m;
    const int m0 = tile_m * BM, n0 = tile_n * BN;
    const size_t kp = (size_t)g.kb * kBlock;

    // a thread's pieces: rows tid / 8 + i * T / 8 of the tile, place tid % 8 in the row
    const uint8_t* src[kRowsA + kRowsB];
#pragma unroll
    for (int i = 0; i < kRowsA + kRowsB; ++i) {
        const bool isa = i < kRowsA;
        const int r = tid / 8 + (isa ? i : i - kRowsA) * (T / 8);
        const int piece = (tid & 7) ^ ((r >> 1) & 7);
        src[i] = isa ? g.a + (size_t)min(m0 + r, g.m - 1) * kp + piece * 16 : g.b + (size_t)min(n0 + r, g.n - 1) * kp + piece * 16;
    }
    auto fetch = [&](int buf, int k) {
#pragma unroll
        for (int i = 0; i < kRowsA + kRowsB; ++i) {
            const int row = (i < kRowsA ? i * (T / 8) : BM + (i - kRowsA) * (T / 8)) + wave * 8;
            __builtin_amdgcn_global_load_lds((global_bytes*)(src[i] + (size_t)k * kBlock), (lds_bytes*)(codes[buf] + row * kBlock), 16, 0, 0);
        }
    };
    auto fetch_scales = [&](int k) {
        for (int r = tid; r < BM + BN; r += T) {
            const uint8_t* row = r < BM ? g.as + (size_t)min(m0 + r, g.m - 1) * g.kb : g.bs + (size_t)min(n0 + r - BM, g.n - 1) * g.kb;
            scales[(k >> 2) & 1][r] = scales_of(row, k, g.kb);
        }
    };
    f32x4 acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = 0.0f;
    uint32_t sa[FM], sb[FN];
    const int fr = lane & 15, q = lane >> 4;
    const int p0 = ((2 * q) ^ ((fr >> 1) & 7)) * 16, p1 = ((2 * q + 1) ^ ((fr >> 1) & 7)) * 16;
    auto fragment = [&](const uint8_t* base, int row) {
        const i32x4 lo = *reinterpret_cast<const i32x4*>(base + row * kBlock + p0), hi = *reinterpret_cast<const i32x4*>(base + row * kBlock + p1);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    fetch(0, 0);
    fetch_scales(0);
    for (int k = 0; k < g.kb; ++k) {
        __builtin_amdgcn_s_waitcnt(0);                         // (the loads that write LDS)
        __syncthreads();
        if (k + 1 < g.kb) {
            fetch((k + 1) & 1, k + 1);
            if (((k + 1) & 3) == 0) fetch_scales(k + 1);
        }
        const uint8_t* buf = codes[k & 1];
        if ((k & 3) == 0) {
#pragma unroll
            for (int j = 0; j < FM; ++j) sa[j] = scales[(k >> 2) & 1][wm * (BM / WM) + j * 16 + fr];
#pragma unroll
            for (int i = 0; i < FN; ++i) sb[i] = scales[(k >> 2) & 1][BM + wn * (BN / WN) + i * 16 + fr];
        }
        typename Operand<kExact>::type fa[FM];
#pragma unroll
        for (int j = 0; j < FM; ++j) fa[j] = operand<kExact>(fragment(buf, wm * (BM / WM) + j * 16 + fr), sa[j]);
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const auto fb = operand<kExact>(fragment(buf + BM * kBlock, wn * (BN / WN) + i * 16 + fr), sb[i]);
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = mfma_blocks(fb, fa[j], acc[i][j], sb[i], sa[j]);
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) sa[j] >>= 8;
#pragma unroll
        for (int i = 0; i < FN; ++i) sb[i] >>= 8;
    }
#pragma unroll
    for (int i = 0; i < FN; ++i) {
        const int col = n0 + wn * (BN / WN) + i * 16 + q * 4;
        const int have = min(4, g.n - col);
        if (have <= 0) continue;
        f32x4 bias = {0.0f, 0.0f, 0.0f, 0.0f};
        if (g.bias) bias = load_piece<float, 4>(g.bias + col, have);
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int row = m0 + wm * (BM / WM) + j * 16 + fr;
            if (row < g.m) store_piece<TY, 4>(static_cast<TY*>(g.out) + (int64_t)row * g.out_stride + col, acc[i][j] + bias, have);
        }
    }
}

}  // namespace
}  // namespace pqt

extern "C" {

size_t pqt_block_product_workspace(int64_t m, int64_t n, int64_t k) {
    (void)m; (void)n; (void)k;
    return 0;
}

int pqt_block_product(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales, int64_t m,
                      int64_t n, int64_t k, const float* bias, void* out, int out_type, int64_t out_stride, void* workspace,
                      size_t workspace_bytes, int device, void* hip_stream) {
    using namespace pqt;
    if (!known_type(out_type)) return fail(PQT_EINVAL, "pqt_block_product: unknown type %d", out_type);
    if (m < 0 || n < 0 || k < 1 || out_stride < n)
        return fail(PQT_EINVAL, "pqt_block_product: m=%lld n=%lld k=%lld stride=%lld out of range", (long long)m, (long long)n, (long long)k, (long long)out_stride);
    if (m > 0x7fffff00 || n > 0x7fffff00 || k > 0x7fffff00)
        return fail(PQT_EUNSUPPORTED, "pqt_block_product: m=%lld n=%lld k=%lld beyond 2^31", (long long)m, (long long)n, (long long)k);
    if (m == 0 || n == 0) return PQT_OK;
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return fail(PQT_EINVAL, "pqt_block_product: null pointer");
    if (!aligned_to(a_codes, 16) || !aligned_to(b_codes, 16) || !aligned_to(out, type_bytes(out_type)) || !aligned_to(bias, 4))
        return fail(PQT_EINVAL, "pqt_block_product: a pointer is not aligned (codes to 16 bytes, the others to their element)");
    const size_t need = pqt_block_product_workspace(m, n, k);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_block_product: workspace of %zu bytes, aligned to 16, needed (%zu given)", need, workspace_bytes);
    ProductArgs g{a_codes, a_scales, b_codes, b_scales, bias, out, out_stride, (int)m, (int)n, (int)((k + kBlock - 1) / kBlock), 0, 0};
    constexpr int BM = 128, BN = 128;
    const int64_t tm = (m + BM - 1) / BM, tn = (n + BN - 1) / BN;
    if (tm * tn > 0xffffff) return fail(PQT_EUNSUPPORTED, "pqt_block_product: %lld x %lld tiles", (long long)tm, (long long)tn);
    g.tiles_m = (int)tm;
    g.tiles_n = (int)tn;
    if (const int rc = check_device(device, "pqt_block_product")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    with_type(out_type, [&](auto y) {
        hipLaunchKernelGGL((product_tile_kernel<decltype(y), BM, BN, 2, 2>), dim3((unsigned)(tm * tn)), dim3(256), 0, st, g);
    });
    HIP_TRY(hipGetLastError());
    return PQT_OK;
}

}  // extern "C"
