// Layer norm of rows, and its gradient.
//
// Forward: a row is read once and stays in registers: a group of lanes -- 8 to 64 for short rows, a workgroup of 256 or 1,024 threads
// for long ones -- holds up to four pieces of eight values a lane, adds them up for the mean, then the squares of their
// distances from it (no difference of large sums), and writes the result.  Weight and bias wait in registers while
// the group walks its rows.  Bound by memory.
//
// Backward: grad and x are read once; two sums over the row (g = grad * weight, and g * h) give dx.  The sums over the rows for
// dweight and dbias are kept in registers too: a group walks rows one grid apart, at the end a workgroup adds its groups' sums in
// LDS and writes one row of each, and columns_kernel adds those rows: no atomics, the same bits on every call.
// One workgroup of 512 threads a compute unit, so that there are few such rows (256: 8 bytes a column and row against 6 bytes an element of
// the input).  Longer rows than one_pass_values() take a kernel for dx and one for the sums.
// In both the next row's values are on their way, as they are, while one is worked on.
//
// Measured (a large copy moves 5.1 TB/s): forward 65,537 x 960 bf16 49 us, 5.2 TB/s; 10,000 x 128 floats 4.5 us.  Backward 16,384 x 4,096 bf16
// 76 us and 5 for the rows of sums, 5.0 TB/s; 4,097 x 1,000 10.8 and 3.9 us, two rows a wavefront: too little on its way (1,024 threads a
// workgroup, whose registers spill: 158 and 18 us a call).
#include "norm.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

struct NormArgs {
    const void* x;
    const void* grad;
    const void* weight;
    const void* bias;
    void* out;                             // y or dx
    float* mean;
    float* rstd;
    float* parts;                          // gradient: workgroups x 2 x D, or null: the one workgroup's sums are ...
    float* dweight;                        // ... these (either may be null)
    float* dbias;
    int64_t rows, x_stride, grad_stride, out_stride;
    int D, param_type, want_parts, stream;
    float eps;
};

template <typename TX, typename TY, int G, int NP>
__global__ __launch_bounds__(G > 256 ? G : 256) void layer_norm_kernel(NormArgs g) {
    constexpr int T = G > 256 ? G : 256, kGroups = T / G;
    constexpr bool kKeep = G * NP <= 2048;     // the longest rows leave no registers for weight and bias: they are read for every row
    __shared__ float scratch[2][16];
    int turn = 0;
    const int l = threadIdx.x & (G - 1);
    const float D = (float)g.D;
    f32x8 w[kKeep ? NP : 1], b[kKeep ? NP : 1];
    int have[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int c = (p * G + l) * kNormE;
        have[p] = max(0, min(kNormE, g.D - c));
        if (!kKeep) continue;
        w[p] = 0.0f;
        b[p] = 0.0f;
        if (have[p]) {
            w[p] = param_piece(g.weight, g.param_type, c, have[p], 1.0f);
            b[p] = param_piece(g.bias, g.param_type, c, have[p], 0.0f);
        }
    }
    typedef typename Piece_<TX, kNormE>::type Raw;
    Raw next[NP];
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            next[p] = Raw{};
            if (have[p] && r < g.rows) next[p] = load_raw<TX, kNormE>(static_cast<const TX*>(g.x) + r * g.x_stride + (p * G + l) * kNormE, have[p]);
        }
    };
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G;
    fetch(r);
    for (; r < g.rows; r += step) {
        f32x8 x[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) x[p] = __builtin_convertvector(next[p], f32x8);
        fetch(r + step);                                       // on its way while this row is worked on
        float s = 0.0f;
#pragma unroll
        for (int p = 0; p < NP; ++p) s += sum8(x[p]);
        const float mean = row_sum<G>(s, scratch, turn) / D;        // (a division: the mean of equal values is that value)
        float q = 0.0f;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            x[p] = x[p] - mean;
#pragma unroll
            for (int j = 0; j < kNormE; ++j) q += j < have[p] ? x[p][j] * x[p][j] : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(row_sum<G>(q, scratch, turn) / D + g.eps);
        TY* dst = static_cast<TY*>(g.out) + r * g.out_stride;
#pragma unroll
        for (int p = 0; p < NP; ++p)
            if (have[p]) {
                const int c = (p * G + l) * kNormE;
                const f32x8 wp = kKeep ? w[kKeep ? p : 0] : param_piece(g.weight, g.param_type, c, have[p], 1.0f);
                const f32x8 bp = kKeep ? b[kKeep ? p : 0] : param_piece(g.bias, g.param_type, c, have[p], 0.0f);
                store_piece<TY, kNormE>(dst + c, x[p] * rstd * wp + bp, have[p], g.stream);
            }
        if (l == 0) {
            if (g.mean) g.mean[r] = mean;
            if (g.rstd) g.rstd[r] = rstd;
        }
    }
}

template <typename T, int G, int NP>
__global__ __launch_bounds__(kGradThreads) void layer_norm_gradient_kernel(NormArgs g) {
    constexpr int kGroups = kGradThreads / G;
    constexpr int kRowsOfSums = kGradThreads / (G < kWave ? kWave : G), kColumns = G * NP * kNormE;
    typedef typename Piece_<T, kNormE>::type Raw;
    __shared__ __align__(16) float sums[kRowsOfSums > 1 ? kRowsOfSums : 1][kRowsOfSums > 1 ? kColumns : 1];
    __shared__ float scratch[2][16];
    int turn = 0;
    const int l = threadIdx.x & (G - 1), group = threadIdx.x / G;
    const float D = (float)g.D;
    f32x8 w[NP], dw[NP], db[NP];
    int have[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int c = (p * G + l) * kNormE;
        have[p] = max(0, min(kNormE, g.D - c));
        w[p] = 0.0f;
        dw[p] = 0.0f;
        db[p] = 0.0f;
        if (have[p]) w[p] = param_piece(g.weight, g.param_type, c, have[p], 1.0f);
    }
    Raw next_x[NP], next_y[NP];
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {      // past the last row: zeros, which add nothing
        const bool mine = r < g.rows;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            next_x[p] = Raw{};
            next_y[p] = Raw{};
            if (have[p] && mine) {
                next_x[p] = load_raw<T, kNormE>(static_cast<const T*>(g.x) + r * g.x_stride + (p * G + l) * kNormE, have[p]);
                next_y[p] = load_raw<T, kNormE>(static_cast<const T*>(g.grad) + r * g.grad_stride + (p * G + l) * kNormE, have[p]);
            }
        }
        next_mean = mine ? g.mean[r] : 0.0f;
        next_rstd = mine ? g.rstd[r] : 0.0f;
    };
    const int64_t step = (int64_t)gridDim.x * kGroups;
    fetch((int64_t)blockIdx.x * kGroups + group);
    // (every group of a workgroup makes as many rounds: there is a barrier in row_sum)
    for (int64_t r0 = (int64_t)blockIdx.x * kGroups; r0 < g.rows; r0 += step) {
        const int64_t r = r0 + group;
        const float mean = next_mean, rstd = next_rstd;
        f32x8 h[NP], y[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            h[p] = up_to((__builtin_convertvector(next_x[p], f32x8) - mean) * rstd, have[p]);
            y[p] = __builtin_convertvector(next_y[p], f32x8);
        }
        fetch(r + step);                                       // on its way while this row is worked on
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            dw[p] = dw[p] + y[p] * h[p];
            db[p] = db[p] + y[p];
            y[p] = y[p] * w[p];
            s1 += sum8(y[p]);
            s2 += sum8(y[p] * h[p]);
        }
        s1 = row_sum<G>(s1, scratch, turn) / D;
        s2 = row_sum<G>(s2, scratch, turn) / D;
        if (r < g.rows) {
            T* dst = static_cast<T*>(g.out) + r * g.out_stride;
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (have[p]) store_piece<T, kNormE>(dst + (p * G + l) * kNormE, (y[p] - s1 - h[p] * s2) * rstd, have[p]);
        }
    }
    if (!g.want_parts) return;
    // The groups' sums, dweight's and then dbias's: over the groups of a wavefront by lanes, over its wavefronts in LDS.
    float* out[2] = {g.dweight, g.dbias};
    if (g.parts) {
        out[0] = g.parts + (size_t)blockIdx.x * 2 * g.D;
        out[1] = out[0] + g.D;
    }
    if constexpr (kRowsOfSums > 1) {
        const int row = threadIdx.x / (G < kWave ? kWave : G);
        for (int round = 0; round < 2; ++round) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                f32x8 v = round ? db[p] : dw[p];
#pragma unroll
                for (int j = 0; j < kNormE; ++j) {
#pragma unroll
                    for (int off = G; off < kWave; off *= 2) v[j] += __shfl_xor(v[j], off, kWave);
                }
                if ((threadIdx.x & (kWave - 1)) < G || G >= kWave) *reinterpret_cast<f32x8*>(&sums[row][(p * G + l) * kNormE]) = v;
            }
            __syncthreads();
            for (int c = threadIdx.x; c < g.D; c += kGradThreads) {
                float v = sums[0][c];
#pragma unroll
                for (int i = 1; i < kRowsOfSums; ++i) v += sums[i][c];
                if (out[round]) out[round][c] = v;
            }
            __syncthreads();
        }
    } else {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int c = (p * G + l) * kNormE;
            if (have[p] && out[0]) store_piece<float, kNormE>(out[0] + c, dw[p], have[p]);
            if (have[p] && out[1]) store_piece<float, kNormE>(out[1] + c, db[p], have[p]);
        }
    }
}

// Rows of more than one_pass_values(), which with the sums of their columns would not fit the registers: dx by a workgroup a row that
// reads it twice, the second time from the caches ...
template <typename T>
__global__ __launch_bounds__(kGradThreads) void long_gradient_kernel(NormArgs g) {
    __shared__ float scratch[2][16];
    int turn = 0;
    const float D = (float)g.D;
    for (int64_t r = blockIdx.x; r < g.rows; r += gridDim.x) {
        const T* xs = static_cast<const T*>(g.x) + r * g.x_stride;
        const T* gs = static_cast<const T*>(g.grad) + r * g.grad_stride;
        T* dst = static_cast<T*>(g.out) + r * g.out_stride;
        const float mean = g.mean[r], rstd = g.rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x * kNormE; c < g.D; c += kGradThreads * kNormE) {
            const int have = min(kNormE, g.D - c);
            const f32x8 y = load_piece<T, kNormE>(gs + c, have) * param_piece(g.weight, g.param_type, c, have, 1.0f);
            s1 += sum8(y);
            s2 += sum8(y * up_to((load_piece<T, kNormE>(xs + c, have) - mean) * rstd, have));
        }
        s1 = row_sum<kGradThreads>(s1, scratch, turn) / D;
        s2 = row_sum<kGradThreads>(s2, scratch, turn) / D;
        for (int c = threadIdx.x * kNormE; c < g.D; c += kGradThreads * kNormE) {
            const int have = min(kNormE, g.D - c);
            const f32x8 y = load_piece<T, kNormE>(gs + c, have) * param_piece(g.weight, g.param_type, c, have, 1.0f);
            const f32x8 h = (load_piece<T, kNormE>(xs + c, have) - mean) * rstd;
            store_piece<T, kNormE>(dst + c, (y - s1 - h * s2) * rstd, have);
        }
    }
}

// ... and the columns' sums of every gridDim.y-th row by a thread for eight columns.
template <typename T>
__global__ __launch_bounds__(256) void long_sums_kernel(NormArgs g) {
    const int c = (blockIdx.x * 256 + threadIdx.x) * kNormE;
    if (c >= g.D) return;
    const int have = min(kNormE, g.D - c);
    f32x8 dw, db;
    dw = 0.0f;
    db = 0.0f;
    for (int64_t r = blockIdx.y; r < g.rows; r += gridDim.y) {
        const f32x8 y = load_piece<T, kNormE>(static_cast<const T*>(g.grad) + r * g.grad_stride + c, have);
        dw = dw + y * ((load_piece<T, kNormE>(static_cast<const T*>(g.x) + r * g.x_stride + c, have) - g.mean[r]) * g.rstd[r]);
        db = db + y;
    }
    float* out = g.parts + (size_t)blockIdx.y * 2 * g.D + c;
    store_piece<float, kNormE>(out, dw, have);
    store_piece<float, kNormE>(out + g.D, db, have);
}

}  // namespace
}  // namespace pqt

extern "C" {

int pqt_layer_norm(const void* x, int type, int64_t rows, int64_t D, int64_t x_stride, const void* weight, const void* bias,
                   int param_type, float eps, void* y, int out_type, int64_t y_stride, float* mean, float* rstd, int device,
                   void* hip_stream) {
    using namespace pqt;
    if (!known_type(type) || !known_type(out_type) || !known_type(param_type))
        return fail(PQT_EINVAL, "pqt_layer_norm: unknown type %d, %d or %d", type, param_type, out_type);
    if (rows < 0 || D < 1 || x_stride < D || y_stride < D || !(eps >= 0.0f))
        return fail(PQT_EINVAL, "pqt_layer_norm: rows=%lld D=%lld strides %lld, %lld eps=%g out of range", (long long)rows, (long long)D,
                    (long long)x_stride, (long long)y_stride, (double)eps);
    if (D > kMaxNormD) return fail(PQT_EUNSUPPORTED, "pqt_layer_norm: D=%lld beyond %lld", (long long)D, (long long)kMaxNormD);
    if (rows == 0) return PQT_OK;
    if (!x || !y) return fail(PQT_EINVAL, "pqt_layer_norm: null pointer");
    if (!aligned_to(x, type_bytes(type)) || !aligned_to(y, type_bytes(out_type)) || !aligned_to(weight, type_bytes(param_type)) ||
        !aligned_to(bias, type_bytes(param_type)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return fail(PQT_EINVAL, "pqt_layer_norm: a pointer is not aligned to its element");
    if (const int rc = check_device(device, "pqt_layer_norm")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    NormArgs g{};
    g.x = x;
    g.weight = weight;
    g.bias = bias;
    g.out = y;
    g.mean = mean;
    g.rstd = rstd;
    g.rows = rows;
    g.x_stride = x_stride;
    g.out_stride = y_stride;
    g.stream = (double)rows * D * type_bytes(out_type) > kStreamBytes;
    g.D = (int)D;
    g.param_type = param_type;
    g.eps = eps;
    with_shape(D, [&](auto G, auto NP) {
        constexpr int kThreads = G.value > 256 ? G.value : 256, kGroups = kThreads / G.value;
        // eight workgroups of 256 threads a compute unit, which then walk the rows
        const unsigned blocks = (unsigned)std::min<int64_t>((rows + kGroups - 1) / kGroups, 2048 * 256 / kThreads);
        with_type(type, [&](auto tx) {
            with_type(out_type, [&](auto ty) {
                hipLaunchKernelGGL((layer_norm_kernel<decltype(tx), decltype(ty), G.value, NP.value>), dim3(blocks), dim3(kThreads), 0, st, g);
            });
        });
    });
    HIP_TRY(hipGetLastError());
    return PQT_OK;
}

size_t pqt_layer_norm_gradient_workspace(int64_t rows, int64_t D) {
    if (rows < 1 || D < 1 || D > pqt::kMaxNormD) return 0;
    return (size_t)std::max(pqt::gradient_blocks(rows, D, PQT_F32), pqt::gradient_blocks(rows, D, PQT_BF16)) * 2 * (size_t)D * sizeof(float);
}

int pqt_layer_norm_gradient(const void* grad, int64_t grad_stride, const void* x, int64_t x_stride, int type, int64_t rows,
                            int64_t D, const void* weight, int param_type, const float* mean, const float* rstd, void* dx,
                            int64_t dx_stride, float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                            int device, void* hip_stream) {
    using namespace pqt;
    if (!known_type(type) || !known_type(param_type)) return fail(PQT_EINVAL, "pqt_layer_norm_gradient: unknown type %d or %d", type, param_type);
    if (rows < 0 || D < 1 || x_stride < D || grad_stride < D || dx_stride < D)
        return fail(PQT_EINVAL, "pqt_layer_norm_gradient: rows=%lld D=%lld strides %lld, %lld, %lld out of range", (long long)rows, (long long)D,
                    (long long)grad_stride, (long long)x_stride, (long long)dx_stride);
    if (D > kMaxNormD) return fail(PQT_EUNSUPPORTED, "pqt_layer_norm_gradient: D=%lld beyond %lld", (long long)D, (long long)kMaxNormD);
    if (rows > 0 && (!grad || !x || !mean || !rstd || !dx)) return fail(PQT_EINVAL, "pqt_layer_norm_gradient: null pointer");
    const size_t eb = type_bytes(type);
    if (!aligned_to(grad, eb) || !aligned_to(x, eb) || !aligned_to(dx, eb) || !aligned_to(weight, type_bytes(param_type)) ||
        !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(dweight, 4) || !aligned_to(dbias, 4))
        return fail(PQT_EINVAL, "pqt_layer_norm_gradient: a pointer is not aligned to its element");
    const bool sums = dweight || dbias;
    const size_t need = sums ? pqt_layer_norm_gradient_workspace(rows, D) : 0;
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_layer_norm_gradient: workspace of %zu bytes, aligned to 16, needed (%zu given)", need, workspace_bytes);
    if (rows == 0 && !sums) return PQT_OK;
    if (const int rc = check_device(device, "pqt_layer_norm_gradient")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    NormArgs g{};
    g.x = x;
    g.grad = grad;
    g.weight = weight;
    g.out = dx;
    g.mean = const_cast<float*>(mean);
    g.rstd = const_cast<float*>(rstd);
    const bool alone = rows > 0 && D <= one_pass_values(type) && gradient_blocks(rows, D, type) == 1;      // (asked for room all the same: that hangs on sizes only)
    g.parts = alone ? nullptr : static_cast<float*>(workspace);
    g.dweight = dweight;
    g.dbias = dbias;
    g.rows = rows;
    g.x_stride = x_stride;
    g.grad_stride = grad_stride;
    g.out_stride = dx_stride;
    g.D = (int)D;
    g.param_type = param_type;
    g.want_parts = sums;
    const unsigned blocks = rows ? gradient_blocks(rows, D, type) : 0;
    if (rows && D > one_pass_values(type)) {
        with_type(type, [&](auto t) {
            hipLaunchKernelGGL((long_gradient_kernel<decltype(t)>), dim3((unsigned)std::min<int64_t>(rows, 2 * kGradBlocks)), dim3(kGradThreads), 0, st, g);
            if (sums)
                hipLaunchKernelGGL((long_sums_kernel<decltype(t)>), dim3((unsigned)((D + 256 * kNormE - 1) / (256 * kNormE)), blocks), dim3(256), 0, st, g);
        });
        HIP_TRY(hipGetLastError());
    } else if (rows) {
        with_gradient_shape(D, [&](auto G, auto NP) {
            with_type(type, [&](auto t) {
                if constexpr (NP.value <= 2 || sizeof(t) == 2)
                    hipLaunchKernelGGL((layer_norm_gradient_kernel<decltype(t), G.value, NP.value>), dim3(blocks), dim3(kGradThreads), 0, st, g);
            });
        });
        HIP_TRY(hipGetLastError());
    }
    if (sums && !alone) {
        hipLaunchKernelGGL(columns_kernel, dim3((unsigned)((2 * D + kWave - 1) / kWave)), dim3(1024), 0, st, g.parts, (int)blocks, (int)(2 * D), (int)D, dweight, dbias);
        HIP_TRY(hipGetLastError());
    }
    return PQT_OK;
}

}  // extern "C"
