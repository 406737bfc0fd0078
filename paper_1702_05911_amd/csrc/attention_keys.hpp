// The kernel of attention's gradient that has keys: dk and dv (attention_gradient.hpp).
#pragma once
#include "attention_gradient.hpp"

namespace pqt {
namespace {

// (four wavefronts a SIMD where 128 registers are enough, three where 168 are)
template <typename T, int DP, int NW, int RT, int BN, bool DIRECT>
__global__ __launch_bounds__(NW* kWave, NW == 4 && sizeof(T) == 2 ? (RT * DP > 64 || (RT == 2 && !DIRECT) ? 2 : RT * DP == 32 ? 4 : 3) : 1) void attention_key_gradient_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * RT * 16, KC = DP / 32, DT = DP / 16;
    typedef Tile<T, BN, DP> QueryTile;
    __shared__ __align__(16) typename QueryTile::S q_0[QueryTile::kSize], q_1[QueryTile::kSize], g_0[QueryTile::kSize], g_1[QueryTile::kSize];
    typedef typename QueryTile::Place Place;
    const QueryTile q_even{(Place)q_0, (int)threadIdx.x & (kWave - 1)}, q_odd{(Place)q_1, (int)threadIdx.x & (kWave - 1)}, g_even{(Place)g_0, (int)threadIdx.x & (kWave - 1)}, g_odd{(Place)g_1, (int)threadIdx.x & (kWave - 1)};
    __shared__ __align__(16) float powers[2][BN], deltas[2][BN];
    __shared__ int large_rows;
    extern __shared__ __align__(16) float room[];
    const int W = most_places<RT, BN>(g.reach);
    const BiasTable table{room, BiasTable::pitch_of(W)};
    int bucket[(2 * most_places<RT, BN>(kMaxReach) + kThreads) / kThreads];
    if (g.bias) BiasTable::look_up<-1, kThreads>(g, W, bucket);
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
        Fragment<T> k[RT][KC], v[RT][KC];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                k[rt][c] = rows_of_memory(static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d, g.k_stride, row0 + rt * 16, len, d, c, lane);
                v[rt][c] = rows_of_memory(static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d, g.v_stride, row0 + rt * 16, len, d, c, lane);
            }
        Loader<T, BN, DP, kThreads, DIRECT> next_q(g.q_stride, d), next_g(g.grad_stride, d);
        if (threadIdx.x == 0) large_rows = 0;                  // (set by lanes of the same wavefront)
        float next_sum = 0.0f, next_delta = 0.0f;
        auto fetch = [&](int at, QueryTile qt, QueryTile gt) __attribute__((always_inline)) {
            const int head = kv * g.group + at / steps, i0 = at % steps * BN;
            next_q.begin(qt, static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, i0, len, d);
            next_g.begin(gt, static_cast<const T*>(g.grad) + r.begin * g.grad_stride + (int64_t)head * d, g.grad_stride, i0, len, d);
            if (threadIdx.x < BN) {
                const int i = i0 + (int)threadIdx.x;
                const int64_t place = (int64_t)head * g.n + r.begin + min(i, len - 1);
                next_sum = i < len ? g.lse_in[place] : -__builtin_inff();
                next_delta = i < len ? g.delta[place] : 0.0f;
            }
        };
        auto arrive = [&](int half, QueryTile qt, QueryTile gt) __attribute__((always_inline)) {
            next_q.finish(qt);
            next_g.finish(gt);
            if (threadIdx.x < BN) {
                powers[half][threadIdx.x] = power_of(next_sum);
                deltas[half][threadIdx.x] = next_delta;
                if (large_sum(next_sum)) large_rows = 1;
            }
        };
        auto step = [&](auto large, LaneOf of, int at, int half, QueryTile qt, QueryTile gt, QueryTile q_next, QueryTile g_next) __attribute__((always_inline)) {
            const int i0 = at % steps * BN;
            if (g.bias && i0 == 0 && at > from) {              // another head's (the last barrier stands after the last reading of the one before)
                table.fill<kThreads>(g, kv * g.group + at / steps, W, min(W, len + M + BN), bucket);
                __syncthreads();
            }
            const bool more = !large.value && at + 1 < to;
            if (more) fetch(at + 1, q_next, g_next);
            const int low = row0 - (i0 + BN - 1), high = row0 + RT * 16 - 1 - i0;      // distances key - query
            const bool near = g.bias && high > -g.reach && low < g.reach;
            const float far = g.bias ? table.v[low >= g.reach ? 0 : 2 * W] : 0.0f;
            const float* bias_at = table.from(i0 + of.quad * 4 - row0 - of.col + W);
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
                    if constexpr (large.value) {
                        const f32x4 top = *reinterpret_cast<const TileFloats*>(reinterpret_cast<TileFloat*>(q_1) + i + of.quad * 4);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][x] = s[rt][x] - top;
                    }
                    const f32x4 power = *reinterpret_cast<const f32x4*>(&powers[half][i + of.quad * 4]);
                    const f32x4 delta = *reinterpret_cast<const f32x4*>(&deltas[half][i + of.quad * 4]);
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
        if (g.bias) table.fill<kThreads>(g, kv * g.group + from / steps, W, min(W, len + M + BN), bucket);
        arrive(0, q_even, g_even);
        __syncthreads();
        for (int at = from; at < to; at += 2) {
            step(std::false_type{}, LaneOf(lane), at, 0, q_even, g_even, q_odd, g_odd);
            if (at + 1 < to) step(std::false_type{}, LaneOf(lane), at + 1, 1, q_odd, g_odd, q_even, g_even);
        }
        if (__builtin_amdgcn_readfirstlane(large_rows)) {      // the second walk: see large_sum()
            const LaneOf of = LaneOf::anew();
            const QueryTile qt{(Place)q_0, of.lane}, gt{(Place)g_0, of.lane};
            if (g.bias) table.fill<kThreads>(g, kv * g.group + from / steps, W, min(W, len + M + BN), bucket);
#pragma nounroll
            for (int at = from; at < to; ++at) {
                fetch(at, qt, gt);
                arrive(0, qt, gt);
                if (threadIdx.x < BN) {
                    const bool has = large_sum(next_sum);      // (of a row that there is)
                    float2 sum = float2{0.0f, __builtin_inff()};
                    if (has) sum = g.large_sums[(int64_t)(kv * g.group + at / steps) * g.n + r.begin + at % steps * BN + (int)threadIdx.x];
                    reinterpret_cast<TileFloat*>(q_1)[threadIdx.x] = sum.x;
                    powers[0][threadIdx.x] = sum.y;
                }
                __syncthreads();
                step(std::true_type{}, of, at, 0, qt, gt, qt, gt);
            }
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

}  // namespace

template <typename T>
void launch_attention_keys(const AttentionArgs& args, int rows, int splits, bool direct, hipStream_t st) {
    with_head(args.d, [&](auto dp) {
        constexpr int DP = dp.value, kQueries = sizeof(T) == 4 && DP > 64 ? 32 : 64;
        auto launch = [&](auto kernel, int waves, int of_workgroup, int most) {
            AttentionArgs g = args;
            g.tiles = g.n / of_workgroup + g.texts + 1;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(g.tiles * (g.heads / g.group)), (unsigned)splits), dim3(waves * kWave), g.bias ? BiasTable::bytes(most) : 0, st, g);
        };
        auto of = [&](auto waves, auto rt, auto step) {
            // (two rows' sums of keys and values of the widest heads leave no registers: 222 spilled.  Heads of 96 spill 8 in bf16 and 26 in f16.)
            constexpr int NW = waves.value, BN = step.value, RT = sizeof(T) * DP > (sizeof(T) == 2 ? 192 : 128) ? 1 : rt.value;
            if (direct) launch(attention_key_gradient_kernel<T, DP, NW, RT, BN, true>, NW, NW * RT * 16, most_places<RT, BN>(args.reach));
            else launch(attention_key_gradient_kernel<T, DP, NW, RT, BN, false>, NW, NW * RT * 16, most_places<RT, BN>(args.reach));
        };
        if (rows == 16) of(Width<1>{}, Width<1>{}, Width<32>{});
        else if (rows == 64) of(Width<4>{}, Width<1>{}, Width<kQueries>{});
        else of(Width<4>{}, Width<2>{}, Width<kQueries>{});
    });
}

}  // namespace pqt
