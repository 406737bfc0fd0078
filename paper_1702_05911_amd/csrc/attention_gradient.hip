// The gradients of attention.  With the weights p_ij = exp(scale q_i . k_j + bias - lse_i) taken again from what the forward pass wrote, delta_i =
// grad_i . out_i and ds_ij = p_ij (grad_i . v_j - delta_i):
//     dq_i = scale sum over j of ds_ij k_j,   dk_j = scale sum over i of ds_ij q_i,   dv_j = sum over i of p_ij grad_i,
//     dbias[head][b] = sum of ds_ij over the distances j - i of bucket b.
//
// Two kernels, so that no sum is anybody else's to add to: one has queries and walks the keys (dq, delta, dbias), one has keys and walks the queries of
// all heads that share them (dk, dv).  Each takes the weights anew, seven products instead of five, and the same inputs give the same bytes.
// As in the forward pass the products are turned so that a lane has one own row, whose weights and ds are the next product's operand where they are.
//
// dbias: a wavefront's ds of 16 queries by 16 keys are added up along their diagonals by moving lanes, so that a lane has one distance, and go to a sum by
// distance in LDS which only this lane's group of sixteen adds to; distances to buckets at the workgroup's end.  Tiles farther away than `reach`
// have one bucket and one sum.
#include "attention.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

// f16: ds, which may be far smaller than f16 numbers reach, are brought to them by a power of two for each own row.  It is chosen from the first ds that
// are not zero, at 2^8, and again when some pass 2^15: what is lost lies 2^-32 below the largest.  (bf16 and fp32 reach as far as the sums do.)
template <typename T>
struct Lift {
    __device__ __forceinline__ float inverse() const { return 1.0f; }
    template <int DT> __device__ __forceinline__ void apply(f32x4&, f32x4&, f32x4 (&)[DT]) {}
};
template <>
struct Lift<Half> {
    float by = 0x1p96f;
    __device__ __forceinline__ float inverse() const { return 1.0f / by; }
    template <int DT>
    __device__ __forceinline__ void apply(f32x4& a, f32x4& b, f32x4 (&sums)[DT]) {
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(a[e]), fabsf(b[e])));
        if (__any(top * by > 0x1p15f)) {
            top = max_of_groups(top);
            if (top * by > 0x1p15f) {
                const uint32_t exponent = __float_as_uint(top) >> 23;
                const float now = exponent < 255 ? __uint_as_float(min(262u - exponent, 254u) << 23) : 1.0f, change = now / by;
#pragma unroll
                for (int x = 0; x < DT; ++x) sums[x] = sums[x] * change;
                by = now;
            }
        }
        a = a * by;
        b = b * by;
    }
};
// what the weights are multiplied by: f16's least normal number is 2^-14, and theirs are at most 1
template <typename T> struct WeightLift { static constexpr float log2 = 0.0f, inverse = 1.0f; };
template <> struct WeightLift<Half> { static constexpr float log2 = 14.0f, inverse = 0x1p-14f; };

template <int N> __device__ __forceinline__ float from_right(float v) { return dpp_move<0x100 + N>(v); }     // of the lane N further, zero past sixteen
template <int N> __device__ __forceinline__ float from_left(float v) { return dpp_move<0x110 + N>(v); }

// the logarithm of the sum as a power of two's; rows without weights have none
__device__ __forceinline__ float power_of(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }

template <typename T, int DP, int NW, int BN, bool WHOLE>
__global__ __launch_bounds__(NW* kWave) void attention_query_gradient_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * 16, KC = DP / 32, DT = DP / 16, kCopies = NW * 4;
    __shared__ __align__(16) Tile<T, BN, DP> ks[2], vs[2];
    __shared__ float table[2 * (kMaxReach + M + BN) + 1];
    __shared__ float far_sums[2][NW];
    extern __shared__ float by_distance[];                     // kCopies x (2 W + 1)
    int64_t t;
    int head;
    place_of_workgroup(g, g.heads, t, head);
    const Rows r = rows_of_workgroup<M>(g, t);
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4, wave = threadIdx.x / kWave;
    T* dq = static_cast<T*>(g.dq) + (int64_t)head * d;
    float* parts = g.parts ? g.parts + (t * g.heads + head) * g.buckets : nullptr;
    if (r.mine && (r.before || !r.text)) {                     // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0;
        clear_rows(dq, g.dq_stride, from, r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span), d);
    }
    const int len = r.len, row0 = r.row0 + wave * 16, row = row0 + col;
    const bool work = r.mine && r.text && r.row0 < len;
    if (!work && parts)
        for (int b = threadIdx.x; b < g.buckets; b += kThreads) parts[b] = 0.0f;
    if (!r.mine || !r.text) return;
    f32x4 sums[DT];
#pragma unroll
    for (int b = 0; b < DT; ++b) sums[b] = f32x4{};
    Lift<T> lift;
    if (work) {
        const int kv = head / g.group;
        const T* k = static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d;
        const T* v = static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d;
        const float cs = g.scale * kLog2e;
        const int W = min(g.reach, len) + M + BN, width = 2 * W + 1;
        if (g.bias) fill_bias<1, kThreads>(g, head, table, W);
        if (parts)
            for (int i = threadIdx.x; i < kCopies * width; i += kThreads) by_distance[i] = 0.0f;
        Fragment<T> q[KC], grad[KC];
        float delta = 0.0f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            q[c] = rows_of_memory(static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, row0, len, d, c);
            grad[c] = rows_of_memory(static_cast<const T*>(g.grad) + r.begin * g.grad_stride + (int64_t)head * d, g.grad_stride, row0, len, d, c);
            const f32x8 o = __builtin_convertvector(
                rows_of_memory(static_cast<const T*>(g.out_in) + r.begin * g.out_stride + (int64_t)head * d, g.out_stride, row0, len, d, c), f32x8);
            const f32x8 y = __builtin_convertvector(grad[c], f32x8) * o;
            delta += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        }
        delta = sum_of_groups(delta);
        const float power = row < len ? power_of(g.lse_in[(int64_t)head * g.n + r.begin + row]) : __builtin_inff();
        if (row < len && quad == 0) g.delta[(int64_t)head * g.n + r.begin + row] = delta;
        float far_left = 0.0f, far_right = 0.0f;
        Loads<T, BN, DP, kThreads, WHOLE> next_k, next_v;
        next_k.fetch(k, g.k_stride, 0, len, d);
        next_v.fetch(v, g.v_stride, 0, len, d);
        next_k.put(ks[0]);
        next_v.put(vs[0]);
        __syncthreads();
        const int steps = (len + BN - 1) / BN;
        float* mine = by_distance + (wave * 4 + quad) * width + W;
        for (int step = 0; step < steps; ++step) {
            const int j0 = step * BN;
            if (step + 1 < steps) {
                next_k.fetch(k, g.k_stride, j0 + BN, len, d);
                next_v.fetch(v, g.v_stride, j0 + BN, len, d);
            }
            const Tile<T, BN, DP>& kt = ks[step & 1];
            const Tile<T, BN, DP>& vt = vs[step & 1];
            const int low = j0 - (row0 + 15), high = j0 + BN - 1 - row0;
            const bool near = g.bias && high > -g.reach && low < g.reach;
            const float far = g.bias && !near ? table[low >= g.reach ? 2 * W : 0] : 0.0f;
            const float* at = table + (j0 + quad * 4 - row0 - col + W);
            float carry = 0.0f;
#pragma unroll
            for (int c = 0; c < BN / 32; ++c) {
                f32x4 s[2], dp[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[h] = f32x4{far, far, far, far};
                    if (near) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[h][e] = at[c * 32 + h * 16 + e];
                    }
                    dp[h] = f32x4{};
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        s[h] = multiply(kt.rows(c * 32 + h * 16, x), q[x], s[h]);
                        dp[h] = multiply(vt.rows(c * 32 + h * 16, x), grad[x], dp[h]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = exp2_of(__builtin_fmaf(s[h][e], cs, -power));
                        s[h][e] = p * (dp[h][e] - delta);
                    }
                    if (j0 + BN > len) {                       // places behind the text's last token
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j0 + c * 32 + h * 16 + quad * 4 + e >= len) s[h][e] = 0.0f;
                    }
                }
                if (parts) {
                    if (near) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // lane `col` gets what lies at key 16 c + 4 quad - col from its query on; what moved past the sixteen lanes is the next sixteen keys'
                            const float sum = ((carry + s[h][0]) + from_right<1>(s[h][1])) + (from_right<2>(s[h][2]) + from_right<3>(s[h][3]));
                            carry = from_left<15>(s[h][1]) + from_left<14>(s[h][2]) + from_left<13>(s[h][3]);
                            mine[j0 + c * 32 + h * 16 + quad * 4 - row0 - col] += sum;
                        }
                    } else {
                        const f32x4 both = s[0] + s[1];
                        const float sum = (both[0] + both[1]) + (both[2] + both[3]);
                        if (low >= g.reach) far_right += sum;
                        else far_left += sum;
                    }
                }
                lift.apply(s[0], s[1], sums);
                const Fragment<T> ds = fragment_of<T>(s[0], s[1]);
#pragma unroll
                for (int b = 0; b < DT; ++b) sums[b] = multiply(kt.columns(c * 32, b), ds, sums[b]);
            }
            if (parts && near) mine[j0 + BN + quad * 4 - row0 - col] += carry;
            if (step + 1 < steps) {
                next_k.put(ks[(step + 1) & 1]);
                next_v.put(vs[(step + 1) & 1]);
            }
            __syncthreads();
        }
        if (parts) {
            far_left = group_sum<kWave>(far_left);
            far_right = group_sum<kWave>(far_right);
            if (lane == 0) {
                far_sums[0][wave] = far_left;
                far_sums[1][wave] = far_right;
            }
            for (int i = threadIdx.x; i < width; i += kThreads) {
                float sum = by_distance[i];
#pragma unroll
                for (int x = 1; x < kCopies; ++x) sum += by_distance[x * width + i];
                by_distance[i] = sum;
                by_distance[width + i] = __int_as_float(g.distances[max(-g.reach, min(i - W, g.reach)) + g.reach]);
            }
            __syncthreads();
            // eight lanes a bucket
            const int first = g.distances[0], last = g.distances[2 * g.reach];
            for (int e = threadIdx.x; e < g.buckets * 8; e += kThreads) {
                const int b = e >> 3;
                float sum = 0.0f;
                for (int i = e & 7; i < width; i += 8) sum += __float_as_int(by_distance[width + i]) == b ? by_distance[i] : 0.0f;
                sum = group_sum<8>(sum);
                if ((e & 7) == 0) {
#pragma unroll
                    for (int w = 0; w < NW; ++w) sum += (first == b ? far_sums[0][w] : 0.0f) + (last == b ? far_sums[1][w] : 0.0f);
                    parts[b] = sum;
                }
            }
        }
    }
    if (row >= r.span) return;
    const float by = g.scale * lift.inverse();
    T* dst = dq + (r.begin + row) * g.dq_stride;
#pragma unroll
    for (int b = 0; b < DT; ++b) {
        const int c = b * 16 + quad * 4;
        store_piece<T, 4>(dst + c, row < len ? sums[b] * by : f32x4{}, d - c);
    }
}

template <typename T, int DP, int NW, int BN, bool WHOLE>
__global__ __launch_bounds__(NW* kWave) void attention_key_gradient_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * 16, KC = DP / 32, DT = DP / 16;
    __shared__ __align__(16) Tile<T, BN, DP> qs[2], gs[2];
    __shared__ __align__(16) float powers[2][BN], deltas[2][BN];
    __shared__ float table[2 * (kMaxReach + M + BN) + 1];
    int64_t t;
    int kv;
    place_of_workgroup(g, g.heads / g.group, t, kv);
    const Rows r = rows_of_workgroup<M>(g, t);
    if (!r.mine) return;
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4, wave = threadIdx.x / kWave;
    T* dk = static_cast<T*>(g.dk) + (int64_t)kv * d;
    T* dv = static_cast<T*>(g.dv) + (int64_t)kv * d;
    if (r.before || !r.text) {                                 // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0, to = r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span);
        clear_rows(dk, g.dk_stride, from, to, d);
        clear_rows(dv, g.dv_stride, from, to, d);
        if (!r.text) return;
    }
    const int len = r.len, row0 = r.row0 + wave * 16, row = row0 + col;
    f32x4 k_sums[DT], v_sums[DT];
#pragma unroll
    for (int b = 0; b < DT; ++b) {
        k_sums[b] = f32x4{};
        v_sums[b] = f32x4{};
    }
    Lift<T> lift;
    if (r.row0 < len) {
        const float cs = g.scale * kLog2e;
        const int W = min(g.reach, len) + M + BN;
        Fragment<T> k[KC], v[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            k[c] = rows_of_memory(static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d, g.k_stride, row0, len, d, c);
            v[c] = rows_of_memory(static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d, g.v_stride, row0, len, d, c);
        }
        Loads<T, BN, DP, kThreads, WHOLE> next_q, next_g;
        float next_power = 0.0f, next_delta = 0.0f;
        // the tiles of all heads one after the other
        auto fetch = [&](int head, int i0) __attribute__((always_inline)) {
            next_q.fetch(static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, i0, len, d);
            next_g.fetch(static_cast<const T*>(g.grad) + r.begin * g.grad_stride + (int64_t)head * d, g.grad_stride, i0, len, d);
            if (threadIdx.x < BN) {
                const int i = i0 + (int)threadIdx.x;
                const int64_t at = (int64_t)head * g.n + r.begin + min(i, len - 1);
                next_power = i < len ? power_of(g.lse_in[at]) : __builtin_inff();
                next_delta = i < len ? g.delta[at] : 0.0f;
            }
        };
        auto put = [&](int half) __attribute__((always_inline)) {
            next_q.put(qs[half]);
            next_g.put(gs[half]);
            if (threadIdx.x < BN) {
                powers[half][threadIdx.x] = next_power;
                deltas[half][threadIdx.x] = next_delta;
            }
        };
        const int steps = (len + BN - 1) / BN;
        int head = kv * g.group, half = 0;
        fetch(head, 0);
        put(0);
        for (int h = 0; h < g.group; ++h, ++head) {
            if (g.bias) fill_bias<-1, kThreads>(g, head, table, W);    // (the last barrier stands after the last reading of it)
            __syncthreads();
            for (int step = 0; step < steps; ++step, half ^= 1) {
                const int i0 = step * BN;
                const bool more = step + 1 < steps || h + 1 < g.group;
                if (step + 1 < steps) fetch(head, i0 + BN);
                else if (more) fetch(head + 1, 0);
                const Tile<T, BN, DP>& qt = qs[half];
                const Tile<T, BN, DP>& gt = gs[half];
                const int low = row0 - (i0 + BN - 1), high = row0 + 15 - i0;       // distances key - query
                const bool near = g.bias && high > -g.reach && low < g.reach;
                const float far = g.bias && !near ? table[low >= g.reach ? 0 : 2 * W] : 0.0f;
                const float* at = table + (i0 + quad * 4 - row0 - col + W);
#pragma unroll
                for (int c = 0; c < BN / 32; ++c) {
                    f32x4 s[2], dp[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int i = c * 32 + x * 16;
                        s[x] = f32x4{far, far, far, far};
                        if (near) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[x][e] = at[i + e];
                        }
                        dp[x] = f32x4{};
#pragma unroll
                        for (int y = 0; y < KC; ++y) {
                            s[x] = multiply(qt.rows(i, y), k[y], s[x]);
                            dp[x] = multiply(gt.rows(i, y), v[y], dp[x]);
                        }
                        const f32x4 power = *reinterpret_cast<const f32x4*>(&powers[half][i + quad * 4]);
                        const f32x4 delta = *reinterpret_cast<const f32x4*>(&deltas[half][i + quad * 4]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[x][e] = exp2_of(__builtin_fmaf(s[x][e], cs, WeightLift<T>::log2 - power[e]));
                            dp[x][e] = s[x][e] * (dp[x][e] - delta[e]);
                        }
                    }
                    const Fragment<T> p = fragment_of<T>(s[0], s[1]);
                    lift.apply(dp[0], dp[1], k_sums);
                    const Fragment<T> ds = fragment_of<T>(dp[0], dp[1]);
#pragma unroll
                    for (int b = 0; b < DT; ++b) {
                        v_sums[b] = multiply(gt.columns(c * 32, b), p, v_sums[b]);
                        k_sums[b] = multiply(qt.columns(c * 32, b), ds, k_sums[b]);
                    }
                }
                if (more) put(half ^ 1);
                __syncthreads();
            }
        }
    }
    if (row >= r.span) return;
    const float by = g.scale * lift.inverse() * WeightLift<T>::inverse;
    T* to_k = dk + (r.begin + row) * g.dk_stride;
    T* to_v = dv + (r.begin + row) * g.dv_stride;
#pragma unroll
    for (int b = 0; b < DT; ++b) {
        const int c = b * 16 + quad * 4;
        store_piece<T, 4>(to_k + c, row < len ? k_sums[b] * by : f32x4{}, d - c);
        store_piece<T, 4>(to_v + c, row < len ? v_sums[b] * WeightLift<T>::inverse : f32x4{}, d - c);
    }
}

// Sums over rows of `columns` values, in a fixed order: 64 columns a workgroup, its sixteen wavefronts a part of the rows each, of every gridDim.y-th
// run of rows; out: gridDim.y x columns.
__global__ __launch_bounds__(1024) void join_kernel(const float* parts, int64_t rows, int64_t columns, float* out) {
    __shared__ float sums[16][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane, per = (rows + gridDim.y - 1) / gridDim.y, from = blockIdx.y * per, to = min(from + per, rows);
    float s = 0.0f;
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
    out[blockIdx.y * columns + c] = s;
}

// Where the workspace's parts begin, in floats.
struct Room { int64_t delta, parts, joined, all; };
inline int gradient_rows(int64_t n, int64_t texts, int heads) { return rows_of_a_workgroup(n, texts, heads) == 16 ? 16 : 64; }
inline int64_t runs_of(int64_t tiles) { return std::min<int64_t>(64, std::max<int64_t>(1, tiles / 256)); }
inline Room room_of(int64_t n, int64_t texts, int heads, int buckets) {
    const int64_t tiles = n / gradient_rows(n, texts, heads) + texts + 1, columns = (int64_t)heads * buckets;
    Room r{};
    r.parts = (heads * n + 3) / 4 * 4;
    r.joined = r.parts + (tiles * columns + 3) / 4 * 4;
    r.all = r.joined + (runs_of(tiles) > 1 ? runs_of(tiles) * columns : 0);
    return r;
}

}  // namespace
}  // namespace pqt

extern "C" {

size_t pqt_attention_gradient_workspace(int64_t n, int64_t texts, int heads, int buckets) {
    using namespace pqt;
    if (n < 1 || texts < 0 || heads < 1 || n > kMaxRows || texts > kMaxRows || heads > 65535) return 0;
    return (size_t)room_of(n, texts, heads, std::max(0, std::min(buckets, kMaxBuckets))).all * sizeof(float);
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
    const size_t need = pqt_attention_gradient_workspace(n, texts, heads, dbias ? buckets : 0);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_attention_gradient: workspace of %zu bytes, aligned to 16, needed (%zu given)", need, workspace_bytes);
    if (n == 0 && !dbias) return PQT_OK;
    if (const int rc = check_device(device, "pqt_attention_gradient")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const int64_t columns = (int64_t)heads * buckets;
    if (n > 0) {
        const Room room = room_of(n, texts, heads, dbias ? buckets : 0);
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
        g.parts = dbias ? at + room.parts : nullptr;
        g.grad_stride = grad_stride;
        g.q_stride = q_stride;
        g.k_stride = k_stride;
        g.v_stride = v_stride;
        g.out_stride = out_stride;
        g.dq_stride = dq_stride;
        g.dk_stride = dk_stride;
        g.dv_stride = dv_stride;
        g.clear = clear;
        const int rows = gradient_rows(n, texts, heads);
        g.tiles = n / rows + texts + 1;
        const unsigned query_blocks = (unsigned)(g.tiles * heads), key_blocks = (unsigned)(g.tiles * kv_heads);
        with_type(type, [&](auto t) {
            typedef decltype(t) T;
            const bool whole = d % (16 / (int)sizeof(T)) == 0;
            with_head(d, [&](auto dp) {
                constexpr int DP = dp.value, kRows = sizeof(T) == 4 && DP > 64 ? 32 : 64;
                auto launch = [&](auto queries, auto keys, int waves, int step) {
                    const size_t bytes = dbias ? sizeof(float) * waves * 4 * (2 * (reach + waves * 16 + step) + 1) : 0;
                    hipLaunchKernelGGL(queries, dim3(query_blocks), dim3(waves * kWave), bytes, st, g);
                    hipLaunchKernelGGL(keys, dim3(key_blocks), dim3(waves * kWave), 0, st, g);
                };
                if (rows == 16)
                    whole ? launch(attention_query_gradient_kernel<T, DP, 1, 32, true>, attention_key_gradient_kernel<T, DP, 1, 32, true>, 1, 32)
                          : launch(attention_query_gradient_kernel<T, DP, 1, 32, false>, attention_key_gradient_kernel<T, DP, 1, 32, false>, 1, 32);
                else
                    whole ? launch(attention_query_gradient_kernel<T, DP, 4, kRows, true>, attention_key_gradient_kernel<T, DP, 4, kRows, true>, 4, kRows)
                          : launch(attention_query_gradient_kernel<T, DP, 4, kRows, false>, attention_key_gradient_kernel<T, DP, 4, kRows, false>, 4, kRows);
            });
        });
        HIP_TRY(hipGetLastError());
        if (dbias) {
            const unsigned runs = (unsigned)runs_of(g.tiles), across = (unsigned)((columns + kWave - 1) / kWave);
            hipLaunchKernelGGL(join_kernel, dim3(across, runs), dim3(1024), 0, st, g.parts, g.tiles, columns, runs > 1 ? at + room.joined : dbias);
            if (runs > 1) hipLaunchKernelGGL(join_kernel, dim3(across), dim3(1024), 0, st, at + room.joined, (int64_t)runs, columns, dbias);
            HIP_TRY(hipGetLastError());
        }
    } else {
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)((columns + kWave - 1) / kWave)), dim3(1024), 0, st, static_cast<const float*>(nullptr), (int64_t)0, columns, dbias);
        HIP_TRY(hipGetLastError());
    }
    return PQT_OK;
}

}  // extern "C"
