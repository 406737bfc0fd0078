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

// dbias adds up ds over all places, where they cancel: what the matrix instruction loses below a sum's last bit has a sign (0.006 of 2^-22 a sum of 64 bf16
// products, 0.04 of f16 ones), and that is what its error came to be (1.2e-6 of it at 64 texts of up to 512 tokens; 3.6e-7 in fp32 throughout).  So every
// other tile multiplies with the gradient's negative.
template <typename T>
__device__ __forceinline__ void negate(Fragment<T>& f) {
    f = __builtin_bit_cast(Fragment<T>, __builtin_bit_cast(u32x4, f) ^ 0x80008000u);
}

template <int N> __device__ __forceinline__ float from_right(float v) { return dpp_move<0x100 + N>(v); }     // of the lane N further, zero past sixteen
template <int N> __device__ __forceinline__ float from_left(float v) { return dpp_move<0x110 + N>(v); }

// the logarithm of the sum as a power of two's; rows without weights have none
__device__ __forceinline__ float power_of(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }
// what weights are to be multiplied by for that power's rounding, the same for all of a row: 1 - rest * ln 2 (the rest is below 2^-13 even of sums of e^1000)
__device__ __forceinline__ float rest_of_power(float lse) {
    const float rest = __builtin_fmaf(lse, kLog2e, -(lse * kLog2e)) + lse * kLog2eRest;
    return fabsf(lse) < __builtin_inff() ? __builtin_fmaf(rest, -kLn2, 1.0f) : 1.0f;
}

// Places of the bias table, and of the sums by distance, on either side: those of the tiles that are near, and sixteen for what is carried past one.
template <int RT, int BN>
__host__ __device__ constexpr int most_places(int reach) { return reach + RT * 16 + BN + 16; }

template <typename T, int DP, int NW, int RT, int BN, bool DIRECT>
__global__ __launch_bounds__(NW* kWave, NW == 4 && sizeof(T) == 2 ? 2 : 1) void attention_query_gradient_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * RT * 16, KC = DP / 32, DT = DP / 16, kCopies = NW * 4;
    typedef Tile<T, BN, DP> KeyTile;
    __shared__ __align__(16) typename KeyTile::S k_0[KeyTile::kSize], k_1[KeyTile::kSize], v_0[KeyTile::kSize], v_1[KeyTile::kSize];
    typedef typename KeyTile::Place Place;
    const KeyTile k_even{(Place)k_0}, k_odd{(Place)k_1}, v_even{(Place)v_0}, v_odd{(Place)v_1};
    __shared__ double far_sums[2][NW];
    extern __shared__ __align__(16) float room[];              // the bias by distance, and kCopies x (2 W + 1) sums
    const BiasTable table{room, BiasTable::pitch_of(most_places<RT, BN>(g.reach))};
    float* const by_distance = room + 4 * table.pitch;
    int64_t t;
    int head;
    place_of_workgroup(g, g.heads, t, head);
    const Rows r = rows_of_workgroup<M>(g, t);
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    T* dq = static_cast<T*>(g.dq) + (int64_t)head * d;
    float* parts = g.parts ? g.parts + (t * g.heads + head) * g.buckets : nullptr;
    if (r.mine && (r.before || !r.text)) {                     // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0;
        clear_rows(dq, g.dq_stride, from, r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span), d);
    }
    const int len = r.len, row0 = r.row0 + wave * RT * 16;
    const bool work = r.mine && r.text && r.row0 < len;
    if (!work && parts)
        for (int b = threadIdx.x; b < g.buckets; b += kThreads) parts[b] = 0.0f;
    if (!r.mine || !r.text) return;
    f32x4 sums[RT][DT];
    Lift<T> lift[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int b = 0; b < DT; ++b) sums[rt][b] = f32x4{};
    if (work) {
        const int kv = head / g.group;
        const T* k = static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d;
        const T* v = static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d;
        const float cs = g.scale * kLog2e;
        const int W = min(most_places<RT, BN>(g.reach), len + M + BN), width = 2 * W + 1;
        Loader<T, BN, DP, kThreads, DIRECT> next_k(g.k_stride, d), next_v(g.v_stride, d);
        next_k.begin(k_even, k, g.k_stride, 0, len, d);
        next_v.begin(v_even, v, g.v_stride, 0, len, d);
        if (g.bias) table.fill<1, kThreads>(g, head, W);
        if (parts)
            for (int i = threadIdx.x; i < kCopies * width; i += kThreads) by_distance[i] = 0.0f;
        Fragment<T> q[RT][KC], grad[RT][KC];
        float delta[RT], power[RT], factor[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = row0 + rt * 16 + col;
            delta[rt] = 0.0f;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                q[rt][c] = rows_of_memory(static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, row0 + rt * 16, len, d, c);
                grad[rt][c] = rows_of_memory(static_cast<const T*>(g.grad) + r.begin * g.grad_stride + (int64_t)head * d, g.grad_stride, row0 + rt * 16, len, d, c);
                const f32x8 o = __builtin_convertvector(
                    rows_of_memory(static_cast<const T*>(g.out_in) + r.begin * g.out_stride + (int64_t)head * d, g.out_stride, row0 + rt * 16, len, d, c), f32x8);
                const f32x8 y = __builtin_convertvector(grad[rt][c], f32x8) * o;
                delta[rt] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
            }
            delta[rt] = sum_of_groups(delta[rt]);
            const float lse = row < len ? g.lse_in[(int64_t)head * g.n + r.begin + row] : -__builtin_inff();
            if (row < len && quad == 0) g.delta[(int64_t)head * g.n + r.begin + row] = delta[rt];
            power[rt] = power_of(lse);
            factor[rt] = rest_of_power(lse);
            delta[rt] *= factor[rt];
        }
        double far_left = 0.0, far_right = 0.0;
        next_k.finish(k_even);
        next_v.finish(v_even);
        __syncthreads();
        const float before = g.bias ? table.v[0] : 0.0f, behind = g.bias ? table.v[2 * W] : 0.0f;
        float* const mine = by_distance + (wave * 4 + quad) * width + W;
        auto step = [&](int j0, KeyTile kt, KeyTile vt, KeyTile k_next, KeyTile v_next) __attribute__((always_inline)) {
            const bool more = j0 + BN < len;
            if (more) {
                next_k.begin(k_next, k, g.k_stride, j0 + BN, len, d);
                next_v.begin(v_next, v, g.v_stride, j0 + BN, len, d);
            }
            const int low = j0 - (row0 + RT * 16 - 1), high = j0 + BN - 1 - row0;
            const bool near = g.bias && high > -g.reach && low < g.reach;
            const float far = low >= g.reach ? behind : before;
            const float* at = table.from(j0 + quad * 4 - row0 - col + W);
            float carry[RT], far_sum = 0.0f;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) carry[rt] = 0.0f;
#pragma unroll
            for (int c = 0; c < BN / 32; ++c) {
                f32x4 s[RT][2], dp[RT][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        s[rt][h] = near ? four_of(at + c * 32 + h * 16 - rt * 16) : f32x4{far, far, far, far};
                        dp[rt][h] = f32x4{};
                    }
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        const Fragment<T> f = kt.rows(c * 32 + h * 16, x);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][h] = multiply(f, q[rt][x], s[rt][h]);
                    }
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        const Fragment<T> f = vt.rows(c * 32 + h * 16, x);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) dp[rt][h] = multiply(f, grad[rt][x], dp[rt][h]);
                    }
                }
                Fragment<T> ds[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[rt][h][e] = exp2_of(__builtin_fmaf(s[rt][h][e], cs, -power[rt])) * __builtin_fmaf(dp[rt][h][e], factor[rt], -delta[rt]);
                        if (j0 + c * 32 + 32 > len) {          // places behind the text's last token
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (j0 + c * 32 + h * 16 + quad * 4 + e >= len) s[rt][h][e] = 0.0f;
                        }
                    }
                    if (parts) {
                        if (near) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                // lane `col` gets what lies at key 16 c + 4 quad - col from its query on; what moved past the sixteen lanes is the next sixteen keys'
                                const f32x4 v = s[rt][h];
                                const float sum = ((carry[rt] + v[0]) + from_right<1>(v[1])) + (from_right<2>(v[2]) + from_right<3>(v[3]));
                                carry[rt] = from_left<15>(v[1]) + from_left<14>(v[2]) + from_left<13>(v[3]);
                                mine[j0 + c * 32 + h * 16 + quad * 4 - (row0 + rt * 16) - col] += sum;
                            }
                        } else {
                            const f32x4 both = s[rt][0] + s[rt][1];
                            far_sum += (both[0] + both[1]) + (both[2] + both[3]);
                        }
                    }
                    lift[rt].apply(s[rt][0], s[rt][1], sums[rt]);
                    ds[rt] = fragment_of<T>(s[rt][0], s[rt][1]);
                }
#pragma unroll
                for (int b = 0; b < DT; ++b) {
                    const Fragment<T> f = kt.columns(c * 32, b);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) sums[rt][b] = multiply(f, ds[rt], sums[rt][b]);
                }
            }
            if (parts) {
                if (near) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) mine[j0 + BN + quad * 4 - (row0 + rt * 16) - col] += carry[rt];
                } else if (low >= g.reach) far_right += far_sum;
                else far_left += far_sum;
            }
            if constexpr (sizeof(T) == 2)
                if (parts)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        factor[rt] = -factor[rt];
#pragma unroll
                        for (int x = 0; x < KC; ++x) negate<T>(grad[rt][x]);
                    }
            if (more) {
                next_k.finish(k_next);
                next_v.finish(v_next);
            }
            __syncthreads();
        };
        for (int j0 = 0; j0 < len; j0 += 2 * BN) {
            step(j0, k_even, v_even, k_odd, v_odd);
            if (j0 + BN < len) step(j0 + BN, k_odd, v_odd, k_even, v_even);
        }
        if (parts) {
#pragma unroll
            for (int off = 1; off < kWave; off *= 2) {
                far_left += __shfl_xor(far_left, off, kWave);
                far_right += __shfl_xor(far_right, off, kWave);
            }
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
                double sum = 0.0;
                for (int i = e & 7; i < width; i += 8) sum += __float_as_int(by_distance[width + i]) == b ? by_distance[i] : 0.0f;
#pragma unroll
                for (int off = 1; off < 8; off *= 2) sum += __shfl_xor(sum, off, kWave);
                if ((e & 7) == 0) {
#pragma unroll
                    for (int w = 0; w < NW; ++w) sum += (first == b ? far_sums[0][w] : 0.0) + (last == b ? far_sums[1][w] : 0.0);
                    parts[b] = (float)sum;
                }
            }
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + rt * 16 + col;
        if (row >= r.span) continue;
        const float by = g.scale * lift[rt].inverse();
        T* dst = dq + (r.begin + row) * g.dq_stride;
#pragma unroll
        for (int b = 0; b < DT; ++b) {
            const int c = b * 16 + quad * 4;
            store_piece<T, 4>(dst + c, row < len ? sums[rt][b] * by : f32x4{}, d - c);
        }
    }
}

template <typename T, int DP, int NW, int RT, int BN, bool DIRECT>
__global__ __launch_bounds__(NW* kWave, NW == 4 && sizeof(T) == 2 ? 2 : 1) void attention_key_gradient_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * RT * 16, KC = DP / 32, DT = DP / 16;
    typedef Tile<T, BN, DP> QueryTile;
    __shared__ __align__(16) typename QueryTile::S q_0[QueryTile::kSize], q_1[QueryTile::kSize], g_0[QueryTile::kSize], g_1[QueryTile::kSize];
    typedef typename QueryTile::Place Place;
    const QueryTile q_even{(Place)q_0}, q_odd{(Place)q_1}, g_even{(Place)g_0}, g_odd{(Place)g_1};
    __shared__ __align__(16) float powers[2][BN], deltas[2][BN];
    extern __shared__ __align__(16) float room[];
    const BiasTable table{room, BiasTable::pitch_of(most_places<RT, BN>(g.reach))};
    int64_t t;
    int kv;
    place_of_workgroup(g, g.heads / g.group, t, kv);
    const Rows r = rows_of_workgroup<M>(g, t);
    if (!r.mine) return;
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int split = blockIdx.y;
    T* dk = static_cast<T*>(g.dk) + (int64_t)kv * d;
    T* dv = static_cast<T*>(g.dv) + (int64_t)kv * d;
    if (r.before || !r.text) {                                 // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0, to = r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span);
        if (split == 0) {
            clear_rows(dk, g.dk_stride, from, to, d);
            clear_rows(dv, g.dv_stride, from, to, d);
        }
        if (!r.text) return;
    }
    const int len = r.len, row0 = r.row0 + wave * RT * 16;
    f32x4 k_sums[RT][DT], v_sums[RT][DT];
    Lift<T> lift[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int b = 0; b < DT; ++b) {
            k_sums[rt][b] = f32x4{};
            v_sums[rt][b] = f32x4{};
        }
    // the tiles of all heads one after the other, of which this workgroup has from .. to - 1
    const int steps = (len + BN - 1) / BN, total = steps * g.group;
    const int from = (int)((int64_t)total * split / gridDim.y), to = (int)((int64_t)total * (split + 1) / gridDim.y);
    if (r.row0 < len && from < to) {
        const float cs = g.scale * kLog2e;
        const int W = min(most_places<RT, BN>(g.reach), len + M + BN);
        Fragment<T> k[RT][KC], v[RT][KC];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                k[rt][c] = rows_of_memory(static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d, g.k_stride, row0 + rt * 16, len, d, c);
                v[rt][c] = rows_of_memory(static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d, g.v_stride, row0 + rt * 16, len, d, c);
            }
        Loader<T, BN, DP, kThreads, DIRECT> next_q(g.q_stride, d), next_g(g.grad_stride, d);
        float next_power = 0.0f, next_delta = 0.0f;
        auto fetch = [&](int at, QueryTile qt, QueryTile gt) __attribute__((always_inline)) {
            const int head = kv * g.group + at / steps, i0 = at % steps * BN;
            next_q.begin(qt, static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, i0, len, d);
            next_g.begin(gt, static_cast<const T*>(g.grad) + r.begin * g.grad_stride + (int64_t)head * d, g.grad_stride, i0, len, d);
            if (threadIdx.x < BN) {
                const int i = i0 + (int)threadIdx.x;
                const int64_t place = (int64_t)head * g.n + r.begin + min(i, len - 1);
                next_power = i < len ? power_of(g.lse_in[place]) : __builtin_inff();
                next_delta = i < len ? g.delta[place] : 0.0f;
            }
        };
        auto arrive = [&](int half, QueryTile qt, QueryTile gt) __attribute__((always_inline)) {
            next_q.finish(qt);
            next_g.finish(gt);
            if (threadIdx.x < BN) {
                powers[half][threadIdx.x] = next_power;
                deltas[half][threadIdx.x] = next_delta;
            }
        };
        auto step = [&](int at, int half, QueryTile qt, QueryTile gt, QueryTile q_next, QueryTile g_next) __attribute__((always_inline)) {
            const int i0 = at % steps * BN;
            if (g.bias && (i0 == 0 || at == from)) {           // another head's (the last barrier stands after the last reading of the one before)
                table.fill<-1, kThreads>(g, kv * g.group + at / steps, W);
                __syncthreads();
            }
            const bool more = at + 1 < to;
            if (more) fetch(at + 1, q_next, g_next);
            const int low = row0 - (i0 + BN - 1), high = row0 + RT * 16 - 1 - i0;      // distances key - query
            const bool near = g.bias && high > -g.reach && low < g.reach;
            const float far = g.bias ? table.v[low >= g.reach ? 0 : 2 * W] : 0.0f;
            const float* bias_at = table.from(i0 + quad * 4 - row0 - col + W);
#pragma unroll
            for (int c = 0; c < BN / 32; ++c) {
                f32x4 s[RT][2], dp[RT][2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int i = c * 32 + x * 16;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        s[rt][x] = near ? four_of(bias_at + i - rt * 16) : f32x4{far, far, far, far};
                        dp[rt][x] = f32x4{};
                    }
#pragma unroll
                    for (int y = 0; y < KC; ++y) {
                        const Fragment<T> f = qt.rows(i, y);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][x] = multiply(f, k[rt][y], s[rt][x]);
                    }
#pragma unroll
                    for (int y = 0; y < KC; ++y) {
                        const Fragment<T> f = gt.rows(i, y);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) dp[rt][x] = multiply(f, v[rt][y], dp[rt][x]);
                    }
                    const f32x4 power = *reinterpret_cast<const f32x4*>(&powers[half][i + quad * 4]);
                    const f32x4 delta = *reinterpret_cast<const f32x4*>(&deltas[half][i + quad * 4]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[rt][x][e] = exp2_of(__builtin_fmaf(s[rt][x][e], cs, WeightLift<T>::log2 - power[e]));
                            dp[rt][x][e] = s[rt][x][e] * (dp[rt][x][e] - delta[e]);
                        }
                }
                Fragment<T> p[RT], ds[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    p[rt] = fragment_of<T>(s[rt][0], s[rt][1]);
                    lift[rt].apply(dp[rt][0], dp[rt][1], k_sums[rt]);
                    ds[rt] = fragment_of<T>(dp[rt][0], dp[rt][1]);
                }
#pragma unroll
                for (int b = 0; b < DT; ++b) {
                    const Fragment<T> fg = gt.columns(c * 32, b), fq = qt.columns(c * 32, b);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        v_sums[rt][b] = multiply(fg, p[rt], v_sums[rt][b]);
                        k_sums[rt][b] = multiply(fq, ds[rt], k_sums[rt][b]);
                    }
                }
            }
            if (more) arrive(half ^ 1, q_next, g_next);
            __syncthreads();
        };
        fetch(from, q_even, g_even);
        arrive(0, q_even, g_even);
        __syncthreads();
        for (int at = from; at < to; at += 2) {
            step(at, 0, q_even, g_even, q_odd, g_odd);
            if (at + 1 < to) step(at + 1, 1, q_odd, g_odd, q_even, g_even);
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + rt * 16 + col;
        if (row >= r.span) continue;
        const float by = g.scale * lift[rt].inverse() * WeightLift<T>::inverse;
        if (gridDim.y > 1) {                                   // this split's part of the sums
            float* part = g.key_parts + (((int64_t)split * (g.heads / g.group) + kv) * g.n + r.begin + row) * (2 * DP) + quad * 4;
#pragma unroll
            for (int b = 0; b < DT; ++b) {
                *reinterpret_cast<f32x4*>(part + b * 16) = k_sums[rt][b] * by;
                *reinterpret_cast<f32x4*>(part + DP + b * 16) = v_sums[rt][b] * WeightLift<T>::inverse;
            }
            continue;
        }
        T* to_k = dk + (r.begin + row) * g.dk_stride;
        T* to_v = dv + (r.begin + row) * g.dv_stride;
#pragma unroll
        for (int b = 0; b < DT; ++b) {
            const int c = b * 16 + quad * 4;
            store_piece<T, 4>(to_k + c, row < len ? k_sums[rt][b] * by : f32x4{}, d - c);
            store_piece<T, 4>(to_v + c, row < len ? v_sums[rt][b] * WeightLift<T>::inverse : f32x4{}, d - c);
        }
    }
}

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

// dk and dv from the parts of shared out queries: a wavefront a row, in the splits' order
template <typename T, int DP>
__global__ __launch_bounds__(256) void key_join_kernel(AttentionArgs g, int splits) {
    int64_t t;
    int kv;
    const int kv_heads = g.heads / g.group;
    place_of_workgroup(g, kv_heads, t, kv);
    const Rows r = rows_of_workgroup<64>(g, t);
    if (!r.mine || !r.text) return;
    const int lane = threadIdx.x & (kWave - 1);
    for (int row = r.row0 + threadIdx.x / kWave; row < min(r.row0 + 64, r.span); row += 256 / kWave) {
        for (int c = lane * 4; c < 2 * DP; c += kWave * 4) {
            f32x4 sum = f32x4{};
            if (row < r.len)
                for (int s = 0; s < splits; ++s)
                    sum = sum + *reinterpret_cast<const f32x4*>(g.key_parts + (((int64_t)s * kv_heads + kv) * g.n + r.begin + row) * (2 * DP) + c);
            const int x = c < DP ? c : c - DP;
            T* to = c < DP ? static_cast<T*>(g.dk) + (r.begin + row) * g.dk_stride : static_cast<T*>(g.dv) + (r.begin + row) * g.dv_stride;
            store_piece<T, 4>(to + (int64_t)kv * g.d + x, sum, g.d - x);
        }
    }
}

// Workgroups' rows and shares, by the sizes alone, and where the workspace's parts begin, in floats.
struct GradientPlan {
    int rows;                              // of a workgroup
    int splits;                            // workgroups that share out a key's queries
    int runs;                              // of the bias' parts that are joined side by side
    int64_t tiles, parts, key_parts, joined, all;
};
inline GradientPlan gradient_plan(int64_t n, int64_t texts, int heads, int kv_heads, int d, int buckets) {
    GradientPlan p{};
    p.rows = rows_of_a_workgroup(n, texts, heads);
    p.tiles = n / p.rows + texts + 1;
    // few workgroups have keys: up to eight share the queries, of which each has four tiles at least
    const int64_t busy = std::max<int64_t>(1, n / p.rows) * kv_heads, of_a_key = (texts ? n / texts : 0) * (heads / kv_heads) / (4 * 64);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, of_a_key), 768 / busy));
    p.runs = (int)std::min<int64_t>(64, std::max<int64_t>(1, p.tiles / 256));
    const int64_t columns = (int64_t)heads * buckets;
    int width = 0;
    with_head(d, [&](auto dp) { width = dp.value; });
    p.parts = (heads * n + 3) / 4 * 4;
    p.key_parts = p.parts + (p.tiles * columns + 3) / 4 * 4;
    p.joined = p.key_parts + (p.splits > 1 ? (int64_t)p.splits * kv_heads * n * 2 * width : 0);
    p.all = p.joined + (p.runs > 1 ? p.runs * columns : 0);
    return p;
}

}  // namespace
}  // namespace pqt

extern "C" {

size_t pqt_attention_gradient_workspace(int64_t n, int64_t texts, int heads, int kv_heads, int d, int buckets) {
    using namespace pqt;
    if (n < 1 || texts < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || d < 1 || d > kMaxHeadD || n > kMaxRows || texts > kMaxRows || heads > 65535) return 0;
    return (size_t)gradient_plan(n, texts, heads, kv_heads, d, std::max(0, std::min(buckets, kMaxBuckets))).all * sizeof(float);
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
    const size_t need = pqt_attention_gradient_workspace(n, texts, heads, kv_heads, d, dbias ? buckets : 0);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(PQT_EINVAL, "pqt_attention_gradient: workspace of %zu bytes, aligned to 16, needed (%zu given)", need, workspace_bytes);
    if (n == 0 && !dbias) return PQT_OK;
    if (const int rc = check_device(device, "pqt_attention_gradient")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const int64_t columns = (int64_t)heads * buckets;
    if (n > 0) {
        const GradientPlan plan = gradient_plan(n, texts, heads, kv_heads, d, dbias ? buckets : 0);
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
        const unsigned query_blocks = (unsigned)(g.tiles * heads);
        with_type(type, [&](auto t) {
            typedef decltype(t) T;
            const bool by_query = direct_rows(k, k_stride, sizeof(T), d) && direct_rows(v, v_stride, sizeof(T), d);
            const bool by_key = direct_rows(q, q_stride, sizeof(T), d) && direct_rows(grad, grad_stride, sizeof(T), d);
            with_head(d, [&](auto dp) {
                constexpr int DP = dp.value, kRows = sizeof(T) == 4 && DP > 64 ? 32 : 64;
                auto launch = [&](auto queries, int waves, int most) {
                    const size_t table = bias ? BiasTable::bytes(most) : 0, sums = dbias ? sizeof(float) * waves * 4 * (2 * most + 1) : 0;
                    hipLaunchKernelGGL(queries, dim3(query_blocks), dim3(waves * kWave), table + sums, st, g);
                };
                auto launch_keys = [&](auto keys, int waves, int rows, int most) {
                    AttentionArgs k = g;
                    k.tiles = n / rows + texts + 1;
                    hipLaunchKernelGGL(keys, dim3((unsigned)(k.tiles * kv_heads), (unsigned)plan.splits), dim3(waves * kWave), bias ? BiasTable::bytes(most) : 0, st, k);
                };
                auto of = [&](auto waves, auto rt, auto step) {
                    // (two rows' sums of keys and values of the widest heads leave no registers: 222 spilled)
                    constexpr int NW = waves.value, RT = rt.value, BN = step.value, KRT = sizeof(T) * DP > (sizeof(T) == 2 ? 192 : 128) ? 1 : RT;
                    const int most = most_places<RT, BN>(reach), key_most = most_places<KRT, BN>(reach);
                    if (by_query) launch(attention_query_gradient_kernel<T, DP, NW, RT, BN, true>, NW, most);
                    else launch(attention_query_gradient_kernel<T, DP, NW, RT, BN, false>, NW, most);
                    if (by_key) launch_keys(attention_key_gradient_kernel<T, DP, NW, KRT, BN, true>, NW, NW * KRT * 16, key_most);
                    else launch_keys(attention_key_gradient_kernel<T, DP, NW, KRT, BN, false>, NW, NW * KRT * 16, key_most);
                };
                if (plan.rows == 16) of(Width<1>{}, Width<1>{}, Width<32>{});
                else if (plan.rows == 64) of(Width<4>{}, Width<1>{}, Width<kRows>{});
                else of(Width<4>{}, Width<2>{}, Width<kRows>{});
                if (plan.splits > 1) {
                    AttentionArgs j = g;
                    j.tiles = n / 64 + texts + 1;
                    hipLaunchKernelGGL((key_join_kernel<T, DP>), dim3((unsigned)(j.tiles * kv_heads)), dim3(256), 0, st, j, plan.splits);
                }
            });
        });
        HIP_TRY(hipGetLastError());
        if (dbias) {
            const unsigned across = (unsigned)((columns + kWave - 1) / kWave);
            hipLaunchKernelGGL(join_kernel, dim3(across, (unsigned)plan.runs), dim3(1024), 0, st, g.parts, g.tiles, columns, plan.runs > 1 ? at + plan.joined : dbias);
            if (plan.runs > 1) hipLaunchKernelGGL(join_kernel, dim3(across), dim3(1024), 0, st, at + plan.joined, (int64_t)plan.runs, columns, dbias);
            HIP_TRY(hipGetLastError());
        }
    } else {
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)((columns + kWave - 1) / kWave)), dim3(1024), 0, st, static_cast<const float*>(nullptr), (int64_t)0, columns, dbias);
        HIP_TRY(hipGetLastError());
    }
    return PQT_OK;
}

}  // extern "C"
