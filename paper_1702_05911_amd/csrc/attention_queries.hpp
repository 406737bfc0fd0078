// The kernel of attention's gradient that has queries: dq, delta and the parts of dbias (attention_gradient.hpp).
#pragma once
#include "attention_gradient.hpp"

namespace pqt {
namespace {

// (three wavefronts a SIMD where 168 registers are enough)
template <typename T, int DP, int NW, int RT, int BN, bool DIRECT, bool RUNS>
__global__ __launch_bounds__(NW* kWave, NW == 4 && sizeof(T) == 2 && RT * DP < 256 ? (RT == 1 && DP <= (DIRECT ? 96 : 64) ? 3 : 2) : 1) void attention_query_gradient_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * RT * 16, KC = DP / 32, DT = DP / 16, kCopies = NW * 4;
    // f16: ds in two parts.  A row's ds cancel in their sum, so that their rounding shows in dq half as much again as dq's own (2,301 and 4,001 tokens, 80 values:
    // 3.1e-4 of dq's size off, its own rounding 2.1e-4; the kernel 217 us, so 258, and by runs of steps 244).  For bf16, and in dk, it shows less: 1.4 times.
    constexpr bool kRest = std::is_same<T, Half>::value;
    typedef Tile<T, BN, DP> KeyTile;
    __shared__ __align__(16) typename KeyTile::S k_0[KeyTile::kSize], k_1[KeyTile::kSize], v_0[KeyTile::kSize], v_1[KeyTile::kSize];
    typedef typename KeyTile::Place Place;
    const KeyTile k_even{(Place)k_0, (int)threadIdx.x & (kWave - 1)}, k_odd{(Place)k_1, (int)threadIdx.x & (kWave - 1)}, v_even{(Place)v_0, (int)threadIdx.x & (kWave - 1)}, v_odd{(Place)v_1, (int)threadIdx.x & (kWave - 1)};
    __shared__ double far_sums[2][NW];
    __shared__ int large_rows[NW];
    extern __shared__ __align__(16) float room[];              // the bias by distance, and kCopies x (2 W + 1) sums
    const int W = most_places<RT, BN>(g.reach), width = sums_pitch(W);
    const BiasTable table{room, BiasTable::pitch_of(W)};
    int bucket[(2 * most_places<RT, BN>(kMaxReach) + kThreads) / kThreads];
    if (g.bias) BiasTable::look_up<1, kThreads>(g, W, bucket);
    float* const by_distance = room + 4 * table.pitch;
    int64_t t;
    int head;
    place_of_workgroup(g, g.heads, t, head);
    const Rows r = rows_of_workgroup<M>(g, t);
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    T* dq = static_cast<T*>(g.dq) + (int64_t)head * d;
    const int distances = 2 * g.reach + 1;
    float* parts = g.parts ? g.parts + (t * g.heads + head) * distances : nullptr;
    if (r.mine && (r.before || !r.text)) {                     // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0;
        clear_rows(dq, g.dq_stride, from, r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span), d);
    }
    const int len = r.len, row0 = r.row0 + wave * RT * 16, S = min(W, len + M + BN);
    const bool work = r.mine && r.text && r.row0 < len;
    if (!work && parts)
        for (int i = threadIdx.x; i < distances; i += kThreads) parts[i] = 0.0f;
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
        Loader<T, BN, DP, kThreads, DIRECT> next_k(g.k_stride, d), next_v(g.v_stride, d);
        next_k.begin(k_even, k, g.k_stride, 0, len, d);
        next_v.begin(v_even, v, g.v_stride, 0, len, d);
        // (of the sums by distance, a short text needs fewer)
        const int first = (W - S) & ~3, pieces = (W + S - first) / 4 + 1;      // of four distances each
        if (parts)
            for (int x = 0; x < kCopies; ++x)
                for (int i = threadIdx.x; i < pieces; i += kThreads) *reinterpret_cast<f32x4*>(&by_distance[x * width + first + 4 * i]) = f32x4{};
        Fragment<T> q[RT][KC], grad[RT][KC];
        float delta[RT], power[RT], factor[RT], sum[RT];
        bool large = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = row0 + rt * 16 + col;
            sum[rt] = row < len ? g.lse_in[(int64_t)head * g.n + r.begin + row] : -__builtin_inff();
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                q[rt][c] = rows_of_memory(static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, row0 + rt * 16, len, d, c, lane);
                grad[rt][c] = rows_of_memory(static_cast<const T*>(g.grad) + r.begin * g.grad_stride + (int64_t)head * d, g.grad_stride, row0 + rt * 16, len, d, c, lane);
            }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = row0 + rt * 16 + col;
            delta[rt] = 0.0f;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const f32x8 o = __builtin_convertvector(
                    rows_of_memory(static_cast<const T*>(g.out_in) + r.begin * g.out_stride + (int64_t)head * d, g.out_stride, row0 + rt * 16, len, d, c, lane), f32x8);
                const f32x8 y = __builtin_convertvector(grad[rt][c], f32x8) * o;
                delta[rt] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
            }
            delta[rt] = sum_of_groups(delta[rt]);
            if (row < len && quad == 0) g.delta[(int64_t)head * g.n + r.begin + row] = delta[rt];
            power[rt] = power_of(sum[rt]);
            factor[rt] = rest_of_power(sum[rt]);
            delta[rt] *= factor[rt];
            large |= large_sum(sum[rt]);
        }
        large = __any(large);
        if (lane == 0) large_rows[wave] = large;
        if (g.bias) table.fill<kThreads>(g, head, W, S, bucket);
        double far_left = 0.0, far_right = 0.0;
        next_k.finish(k_even);
        next_v.finish(v_even);
        __syncthreads();
        const float before = g.bias ? table.v[0] : 0.0f, behind = g.bias ? table.v[2 * W] : 0.0f;
        auto step = [&](auto kind, LaneOf of, int j0, KeyTile kt, KeyTile vt, KeyTile k_next, KeyTile v_next) __attribute__((always_inline)) {
            constexpr int kKind = decltype(kind)::value;
            const int lane = of.lane, col = of.col, quad = of.quad;
            float* const mine = by_distance + (wave * 4 + quad) * width + W;
            if constexpr (kKind < kLast) {
                next_k.begin(k_next, k, g.k_stride, j0 + BN, len, d);
                next_v.begin(v_next, v, g.v_stride, j0 + BN, len, d);
            }
            const int low = j0 - (row0 + RT * 16 - 1), high = j0 + BN - 1 - row0;
            const bool near = kKind == kNear || (kKind != kFar && g.bias && high > -g.reach && low < g.reach);
            const float far = low >= g.reach ? behind : before;
            const f32x4 all_far = f32x4{far, far, far, far};
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
                        if constexpr (kKind != kFar) s[rt][h] = near ? four_of(at + c * 32 + h * 16 - rt * 16) : all_far;
                        dp[rt][h] = f32x4{};
                    }
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        const Fragment<T> f = kt.rows(c * 32 + h * 16, x);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][h] = multiply(f, q[rt][x], kKind == kFar && x == 0 ? all_far : s[rt][h]);
                    }
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        const Fragment<T> f = vt.rows(c * 32 + h * 16, x);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) dp[rt][h] = multiply(f, grad[rt][x], dp[rt][h]);
                    }
                }
                Fragment<T> ds[RT], rest[kRest ? RT : 1];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if constexpr (kKind == kLarge) s[rt][h] = s[rt][h] - reinterpret_cast<TileFloat*>(k_1)[(wave * RT + rt) * 16 + col];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[rt][h][e] = exp2_of(__builtin_fmaf(s[rt][h][e], cs, -power[rt])) * __builtin_fmaf(dp[rt][h][e], factor[rt], -delta[rt]);
                        if constexpr (kKind >= kLast) {        // places behind the text's last token
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[rt][h][e] = j0 + c * 32 + h * 16 + quad * 4 + e < len ? s[rt][h][e] : 0.0f;
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
                                add_to(mine + j0 + c * 32 + h * 16 + quad * 4 - (row0 + rt * 16) - col, sum);
                            }
                        } else {
                            const f32x4 both = s[rt][0] + s[rt][1];
                            far_sum += (both[0] + both[1]) + (both[2] + both[3]);
                        }
                    }
                    lift[rt].apply(s[rt][0], s[rt][1], sums[rt]);
                    ds[rt] = fragment_of<T>(s[rt][0], s[rt][1]);
                    if constexpr (kRest) {
                        const f32x8 kept = __builtin_convertvector(ds[rt], f32x8);
                        rest[rt] = fragment_of<T>(s[rt][0] - __builtin_shufflevector(kept, kept, 0, 1, 2, 3), s[rt][1] - __builtin_shufflevector(kept, kept, 4, 5, 6, 7));
                    }
                }
#pragma unroll
                for (int b = 0; b < DT; ++b) {
                    const Fragment<T> f = kt.columns(c * 32, b);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        sums[rt][b] = multiply(f, ds[rt], sums[rt][b]);
                        if constexpr (kRest) sums[rt][b] = multiply(f, rest[rt], sums[rt][b]);
                    }
                }
            }
            if (parts) {
                if (near) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) add_to(mine + j0 + BN + quad * 4 - (row0 + rt * 16) - col, carry[rt]);
                } else if (low >= g.reach) far_right += far_sum;
                else far_left += far_sum;
            }
            if constexpr (kKind < kLast) {
                if constexpr (sizeof(T) == 2) {
                    if (parts) {
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            factor[rt] = -factor[rt];
#pragma unroll
                            for (int x = 0; x < KC; ++x) negate<T>(grad[rt][x]);
                        }
                    }
                }
                next_k.finish(k_next);
                next_v.finish(v_next);
            }
            __syncthreads();
        };
        walk<RT, BN, RUNS>(g, row0, len, [&](auto kind, auto odd, int i) __attribute__((always_inline)) {
            if constexpr (odd.value) step(kind, LaneOf(lane), i * BN, k_odd, v_odd, k_even, v_even);
            else step(kind, LaneOf(lane), i * BN, k_even, v_even, k_odd, v_odd);
        });
        large = false;
#pragma unroll
        for (int w = 0; w < NW; ++w) large |= large_rows[w] != 0;
        if (__builtin_amdgcn_readfirstlane(large)) {           // the second walk: see large_sum()
            const LaneOf of = LaneOf::anew();
            const int lane = of.lane, col = of.col, quad = of.quad;
            const KeyTile kt{(Place)k_0, lane}, vt{(Place)v_0, lane};
            // maxima and sums, by products that start as the steps' do
            float most[RT], total[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                most[rt] = kLowest;
                total[rt] = 0.0f;
            }
#pragma nounroll
            for (int j0 = 0; j0 < len; j0 += 16) {
                const int tile = j0 - j0 % BN, low = tile - (row0 + RT * 16 - 1), high = tile + BN - 1 - row0;
                const bool near = g.bias && high > -g.reach && low < g.reach;
                const float far = low >= g.reach ? behind : before;
                const float* at = table.from(j0 + quad * 4 - row0 - col + W);
                f32x4 s[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt] = near ? four_of(at - rt * 16) : f32x4{far, far, far, far};
#pragma unroll
                for (int x = 0; x < KC; ++x) {
                    const Fragment<T> f = rows_of_memory(k, g.k_stride, j0, len, d, x, lane);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt] = multiply(f, q[rt][x], s[rt]);
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[rt][e] = j0 + quad * 4 + e < len ? s[rt][e] : -__builtin_inff();
                    const float now = fmaxf(fmaxf(fmaxf(most[rt], s[rt][0]), fmaxf(s[rt][1], s[rt][2])), s[rt][3]);
                    total[rt] *= exp2_of((most[rt] - now) * cs);
                    most[rt] = now;
#pragma unroll
                    for (int e = 0; e < 4; ++e) total[rt] += exp2_of((s[rt][e] - now) * cs);
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int row = row0 + rt * 16 + col;
                const int64_t place = (int64_t)head * g.n + r.begin + row;
                const bool has = row < len && large_sum(g.lse_in[place]);
                const float top = max_of_groups(most[rt]);
                power[rt] = has ? __builtin_amdgcn_logf(sum_of_groups(total[rt] * exp2_of((most[rt] - top) * cs))) : __builtin_inff();
                reinterpret_cast<TileFloat*>(k_1)[(wave * RT + rt) * 16 + col] = has ? top : 0.0f;
                if (has && quad == 0) g.large_sums[place] = float2{top, power[rt]};
            }
#pragma nounroll
            for (int j0 = 0; j0 < len; j0 += BN) {
                next_k.begin(kt, k, g.k_stride, j0, len, d);
                next_v.begin(vt, v, g.v_stride, j0, len, d);
                next_k.finish(kt);
                next_v.finish(vt);
                __syncthreads();
                step(Kind<kLarge>{}, of, j0, kt, vt, kt, vt);
            }
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
            // The sums of the distances nearer than `reach`; what lies farther has its ends' buckets and is added up.
            for (int i = threadIdx.x; i < pieces; i += kThreads) {
                float* const to = by_distance + first + 4 * i;
                f32x4 sum = four_of(to);
#pragma unroll
                for (int x = 1; x < kCopies; ++x) sum = sum + four_of(to + x * width);
                *reinterpret_cast<f32x4*>(to) = sum;
            }
            __syncthreads();
            for (int i = threadIdx.x + 1; i < distances - 1; i += kThreads) {
                const int at = i - g.reach;
                parts[i] = at >= -S && at <= S ? by_distance[W + at] : 0.0f;
            }
            for (int side = wave; side < 2; side += NW) {
                double sum = 0.0;
                for (int at = g.reach + lane; at <= S; at += kWave) sum += by_distance[W + (side ? at : -at)];
#pragma unroll
                for (int off = 1; off < kWave; off *= 2) sum += __shfl_xor(sum, off, kWave);
#pragma unroll
                for (int w = 0; w < NW; ++w) sum += far_sums[side][w];
                // (a reach of 0 has one bucket, both sides' and the middle's: the middle counts once)
                if (g.reach > 0) {
                    if (lane == 0) parts[side ? distances - 1 : 0] = (float)sum;
                } else if (side == 0) {
                    double right = 0.0;
                    for (int at = 1 + lane; at <= S; at += kWave) right += by_distance[W + at];
#pragma unroll
                    for (int off = 1; off < kWave; off *= 2) right += __shfl_xor(right, off, kWave);
#pragma unroll
                    for (int w = 0; w < NW; ++w) right += far_sums[1][w];
                    if (lane == 0) parts[0] = (float)(sum + right);
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

}  // namespace

template <typename T>
void launch_attention_queries(const AttentionArgs& args, int rows, bool direct, hipStream_t st) {
    AttentionArgs g = args;
    g.tiles = g.n / rows + g.texts + 1;
    const dim3 blocks((unsigned)(g.tiles * g.heads));
    with_head(g.d, [&](auto dp) {
        constexpr int DP = dp.value, kKeys = sizeof(T) == 4 && DP > 64 ? 32 : 64;
        auto launch = [&](auto kernel, int waves, int most) {
            const size_t table = g.bias ? BiasTable::bytes(most) : 0, sums = g.parts ? sizeof(float) * waves * 4 * sums_pitch(most) : 0;
            hipLaunchKernelGGL(kernel, blocks, dim3(waves * kWave), table + sums, st, g);
        };
        auto of = [&](auto waves, auto rt, auto step, auto runs) {
            constexpr int NW = waves.value, RT = rt.value, BN = step.value;
            if (direct) launch(attention_query_gradient_kernel<T, DP, NW, RT, BN, true, runs.value>, NW, most_places<RT, BN>(g.reach));
            else launch(attention_query_gradient_kernel<T, DP, NW, RT, BN, false, false>, NW, most_places<RT, BN>(g.reach));
        };
        typedef std::integral_constant<bool, false> No;
        typedef std::integral_constant<bool, true> Yes;
        if (rows == 16) of(Width<1>{}, Width<1>{}, Width<32>{}, No{});
        else if (rows == 64) of(Width<4>{}, Width<1>{}, Width<kKeys>{}, No{});
        else if (!long_texts(g.n, g.texts)) of(Width<4>{}, Width<2>{}, Width<kKeys>{}, No{});
        // (at heads of 96 runs spill 62 registers, f16's two parts of ds 75, and pay all the same: four texts of 4,096 tokens, 16 heads, without and with runs bf16 1,720 and 1,641 us, f16 2,120 and 2,041;
        // two of 3,150, 8 heads of 80, 359 and 345, 438 and 425; 16 of 1,100, 12 heads of 96, 567 and 585, 691 and 712)
        else of(Width<4>{}, Width<2>{}, Width<kKeys>{}, Yes{});
    });
}

}  // namespace pqt
