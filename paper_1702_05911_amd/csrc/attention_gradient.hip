// Attention's gradient: the C entry, the plan of its kernels, and the sums of what they leave in parts.
#include "attention.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

// Sums over rows of `columns` values, in 64 bits and a fixed order: 64 columns a workgroup, its sixteen wavefronts a part of the rows each, of every gridDim.y-th
// run of rows; out: gridDim.y x columns.
__global__ __launch_bounds__(1024) void join_kernel(const float* parts, int64_t rows, int64_t columns, float* out) {
    __shared__ double sums[16][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane, per = (rows + gridDim.y - 1) / gridDim.y, from = blockIdx.y * per, to = min(from + per, rows);
    double s = 0.0;
    if (c < columns)
        for (int64_t r = from + wave; r < to; r += 16 * 8) {   // eight rows on their way
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = parts[min(r + 16 * u, to - 1) * columns + c];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += r + 16 * u < to ? v[u] : 0.0f;
        }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= columns) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    out[blockIdx.y * columns + c] = (float)s;
}

// dbias: a workgroup a head adds up `rows` parts (or joined parts) of every distance, every fourth by a quarter of its threads, and then the distances of every
// bucket, eight lanes each; in 64 bits and a fixed order.
__global__ __launch_bounds__(1024) void bucket_kernel(const float* parts, int rows, AttentionArgs g, float* dbias) {
    __shared__ double sums[4][2 * kMaxReach + 1];
    __shared__ int bucket[2 * kMaxReach + 1];
    const int distances = 2 * g.reach + 1, quarter = threadIdx.x >> 8;
    for (int i = threadIdx.x & 255; i < distances; i += 256) {
        if (quarter == 0) bucket[i] = g.distances[i];
        double s = 0.0;
        for (int r0 = quarter; r0 < rows; r0 += 4 * 16) {      // sixteen on their way
            float v[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = parts[((int64_t)min(r0 + 4 * u, rows - 1) * g.heads + blockIdx.x) * distances + i];
#pragma unroll
            for (int u = 0; u < 16; ++u) s += r0 + 4 * u < rows ? v[u] : 0.0f;
        }
        sums[quarter][i] = s;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < distances; i += 1024) sums[0][i] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    __syncthreads();
    for (int e = threadIdx.x; e < g.buckets * 8; e += 1024) {
        double s = 0.0;
#pragma unroll 8
        for (int i = e & 7; i < distances; i += 8) s += bucket[i] == e >> 3 ? sums[0][i] : 0.0;
#pragma unroll
        for (int off = 1; off < 8; off *= 2) s += __shfl_xor(s, off, kWave);
        if ((e & 7) == 0) dbias[(int64_t)blockIdx.x * g.buckets + (e >> 3)] = (float)s;
    }
}

// dk and dv from the parts of shared out queries, four values a thread at a time, in the splits' order
template <typename T, int DP>
__global__ __launch_bounds__(256) void key_join_kernel(AttentionArgs g, int splits) {
    int64_t t;
    int kv;
    const int kv_heads = g.heads / g.group;
    place_of_workgroup(g, kv_heads, t, kv);
    const Rows r = rows_of_workgroup<64>(g, t);
    if (!r.mine || !r.text) return;
    const int rows = min(64, r.span - r.row0);
    const int64_t apart = (int64_t)kv_heads * g.n * (2 * DP);
    for (int e = threadIdx.x; e < rows * (2 * DP / 4); e += 256) {
        const int row = r.row0 + e / (2 * DP / 4), c = e % (2 * DP / 4) * 4, x = c < DP ? c : c - DP;
        if (x >= g.d) continue;
        f32x4 sum = f32x4{};
        if (row < r.len) {
            const float* part = g.key_parts + ((int64_t)kv * g.n + r.begin + row) * (2 * DP) + c;
#pragma unroll 4
            for (int s = 0; s < splits; ++s) sum = sum + *reinterpret_cast<const f32x4*>(part + s * apart);
        }
        T* to = c < DP ? static_cast<T*>(g.dk) + (r.begin + row) * g.dk_stride : static_cast<T*>(g.dv) + (r.begin + row) * g.dv_stride;
        store_piece<T, 4>(to + (int64_t)kv * g.d + x, sum, g.d - x);
    }
}

// Workgroups' rows and shares, by the sizes alone, and where the workspace's parts begin, in floats.
struct GradientPlan {
    int rows;                              // of a workgroup
    int splits;                            // workgroups that share out a key's queries
    int runs;                              // of the bias' parts that are joined side by side; 0: few parts, none are
    int64_t tiles, large_sums, parts, key_parts, joined, all;
};
// (reach: -1 where there is no dbias)
inline GradientPlan gradient_plan(int64_t n, int64_t texts, int heads, int kv_heads, int d, int reach) {
    GradientPlan p{};
    // 16 where texts are short (16 heads of 64 bf16 values, 16 and 64 rows: 3,000 texts of 20 tokens 1,191 and 1,302 us, 2,048 of 32 934 and 978, 1,800 of 36 1,213 and 910)
    p.rows = texts && n / texts <= 32 ? 16 : rows_of_a_workgroup(n, texts, heads);
    p.tiles = n / p.rows + texts + 1;
    int width = 0;
    with_head(d, [&](auto dp) { width = dp.value; });
    // Few workgroups have keys: up to eight share the queries, of which each has four tiles at least.  As many as make the time least, counted in rounds of what the
    // card holds at once, four fifths of it: a round that is all but full leaves a shader engine with a workgroup too many, for which it waits.  (Heads of 64 bf16
    // values, 16 of them: one text of 4,000, two of keys, shared by one 1,086 us, 4 427, 6 336, 8 392; two such 1,187, 3 632, 4 743, 6 624; one of 1,000, four of keys, 64 rows 130, 4 76, 8 70.
    // Two texts of 3,150, 8 heads of 80 f16 values, two of keys: 4 395, 6 436, 8 403.)
    const int key_rows = width > 96 ? std::min(p.rows, 64) : p.rows, at_once = key_rows <= 64 && width <= 64 ? 800 : 400;
    const int64_t busy = std::max<int64_t>(1, n / key_rows) * kv_heads, most = std::min<int64_t>(std::min<int64_t>(8, (texts ? n / texts : 0) * (heads / kv_heads) / (4 * 64)), 800 / busy);
    p.splits = 1;
    int64_t rounds = (busy + at_once - 1) / at_once;
    for (int s = 2; s <= most; ++s) {
        const int64_t r = (busy * s + at_once - 1) / at_once;
        if (r * p.splits < rounds * s) {
            p.splits = s;
            rounds = r;
        }
    }
    p.runs = p.tiles > 64 ? (int)std::min<int64_t>(64, p.tiles / 32) : 0;
    const int64_t columns = (int64_t)heads * (2 * reach + 1);
    const bool sums = reach >= 0;
    p.large_sums = (heads * n + 3) / 4 * 4;
    p.parts = p.large_sums + (2 * heads * n + 3) / 4 * 4;
    p.key_parts = p.parts + (sums ? (p.tiles * columns + 3) / 4 * 4 : 0);
    p.joined = p.key_parts + (p.splits > 1 ? (int64_t)p.splits * kv_heads * n * 2 * width : 0);
    p.all = p.joined + (sums ? p.runs * columns : 0);
    return p;
}

}  // namespace
}  // namespace pqt

extern "C" {

size_t pqt_attention_gradient_workspace(int64_t n, int64_t texts, int heads, int kv_heads, int d, int reach) {
    using namespace pqt;
    if (n < 1 || texts < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || d < 1 || d > kMaxHeadD || n > kMaxRows || texts > kMaxRows || heads > 65535) return 0;
    return (size_t)gradient_plan(n, texts, heads, kv_heads, d, std::max(-1, std::min(reach, kMaxReach))).all * sizeof(float);
}

int pqt_attention_gradient(const void* grad, int64_t grad_stride, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                           int64_t v_stride, const void* out, int64_t out_stride, const float* lse, int type, int64_t n, int heads, int kv_heads, int d,
                           const void* starts, const void* lengths, int place_bytes, int64_t texts, float scale, const float* bias, int buckets,
                           const int32_t* distances, int reach, int clear, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, void* dv,
                           int64_t dv_stride, float* dbias, void* workspace, size_t workspace_bytes, int device, void* hip_stream) {
    using namespace pqt;
    AttentionArgs g{};
    if (const int rc = attention_checks("pqt_attention_gradient", type, n, heads, kv_heads, d, starts, lengths, place_bytes, texts, scale, bias, buckets, distances, reach, g)) return rc;
    const int64_t wide = (int64_t)heads * d, narrow = (int64_t)kv_heads * d;
    if (grad_stride < wide || q_stride < wide || k_stride < narrow || v_stride < narrow || out_stride < wide || dq_stride < wide || dk_stride < narrow || dv_stride < narrow)
        return fail(PQT_EINVAL, "pqt_attention_gradient: a stride below the %lld values of a row (of keys %lld)", (long long)wide, (long long)narrow);
    if (dbias && !bias) return fail(PQT_EINVAL, "pqt_attention_gradient: the gradient of a bias that is not there");
    if (n > 0 && (!grad || !q || !k || !v || !out || !lse || !dq || !dk || !dv)) return fail(PQT_EINVAL, "pqt_attention_gradient: null pointer");
    const size_t eb = type_bytes(type);
    if (!aligned_to(grad, eb) || !aligned_to(q, eb) || !aligned_to(k, eb) || !aligned_to(v, eb) || !aligned_to(out, eb) || !aligned_to(dq, eb) || !aligned_to(dk, eb) ||
        !aligned_to(dv, eb) || !aligned_to(lse, 4) || !aligned_to(dbias, 4))
        return fail(PQT_EINVAL, "pqt_attention_gradient: a pointer is not aligned to its element");
    const size_t need = pqt_attention_gradient_workspace(n, texts, heads, kv_heads, d, dbias ? reach : -1);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_attention_gradient: workspace of %zu bytes, aligned to 16, needed (%zu given)", need, workspace_bytes);
    if (n == 0 && !dbias) return PQT_OK;
    if (const int rc = check_device(device, "pqt_attention_gradient")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (n > 0) {
        const GradientPlan plan = gradient_plan(n, texts, heads, kv_heads, d, dbias ? reach : -1);
        float* const at = static_cast<float*>(workspace);
        g.grad = grad;
        g.q = q;
        g.k = k;
        g.v = v;
        g.out_in = out;
        g.lse_in = lse;
        g.dq = dq;
        g.dk = dk;
        g.dv = dv;
        g.delta = at;
        g.large_sums = reinterpret_cast<float2*>(at + plan.large_sums);
        g.parts = dbias ? at + plan.parts : nullptr;
        g.key_parts = at + plan.key_parts;
        g.grad_stride = grad_stride;
        g.q_stride = q_stride;
        g.k_stride = k_stride;
        g.v_stride = v_stride;
        g.out_stride = out_stride;
        g.dq_stride = dq_stride;
        g.dk_stride = dk_stride;
        g.dv_stride = dv_stride;
        g.clear = clear;
        g.tiles = plan.tiles;
        with_type(type, [&](auto t) {
            typedef decltype(t) T;
            launch_attention_queries<T>(g, plan.rows, direct_rows(k, k_stride, sizeof(T), d) && direct_rows(v, v_stride, sizeof(T), d), st);
            launch_attention_keys<T>(g, plan.rows, plan.splits, direct_rows(q, q_stride, sizeof(T), d) && direct_rows(grad, grad_stride, sizeof(T), d), st);
            if (plan.splits > 1)
                with_head(d, [&](auto dp) {
                    AttentionArgs j = g;
                    j.tiles = n / 64 + texts + 1;
                    hipLaunchKernelGGL((key_join_kernel<T, dp.value>), dim3((unsigned)(j.tiles * kv_heads)), dim3(256), 0, st, j, plan.splits);
                });
        });
        HIP_TRY(hipGetLastError());
        if (dbias) {
            const int64_t columns = (int64_t)heads * (2 * reach + 1);
            if (plan.runs)
                hipLaunchKernelGGL(join_kernel, dim3((unsigned)((columns + kWave - 1) / kWave), (unsigned)plan.runs), dim3(1024), 0, st, g.parts, g.tiles, columns, at + plan.joined);
            hipLaunchKernelGGL(bucket_kernel, dim3((unsigned)heads), dim3(1024), 0, st, plan.runs ? at + plan.joined : g.parts, plan.runs ? plan.runs : (int)g.tiles, g, dbias);
            HIP_TRY(hipGetLastError());
        }
    } else {
        hipLaunchKernelGGL(bucket_kernel, dim3((unsigned)heads), dim3(1024), 0, st, static_cast<const float*>(nullptr), 0, g, dbias);
        HIP_TRY(hipGetLastError());
    }
    return PQT_OK;
}

}  // extern "C"
