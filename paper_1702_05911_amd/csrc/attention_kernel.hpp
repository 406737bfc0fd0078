// The kernel of attention among the tokens of every text: out_i = sum over j of p_ij v_j, p_ij = softmax over j of scale q_i . k_j + bias[bucket of j - i].
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup has 64 or 128 queries of one head, a wavefront one or two times 16
// of them, in registers; tiles of keys and values go through LDS in turn, two of each, the next one on its way from memory.  Products are
// taken transposed -- keys by queries, then values' columns by queries -- so that a lane has one query's logits, and the weights become the second
// product's operand where they are.
//
// Long texts are bound by the vector and the matrix unit in turn: a weight is a multiplication and addition, a power of two, a sum and a conversion, for 4 d operations of
// products, and each unit is busy for half of the time (one text of 8,191 tokens, 16 heads of 128 bf16 values, four of keys: 508 us, 1.08 PFLOP/s where a large library
// product makes 1.6; its kernel spills 46 registers, none of them within a run of steps).  Shorter ones wait for their first loads and last stores: 512 texts of up to 256, 12 heads of 64, 201 us,
// 555 MB at 2.8 TB/s, vector unit 57 % of the time, matrix unit 13 %, 41 % of the wavefronts' time waiting.
#pragma once
#include "attention.hpp"

namespace pqt {
namespace {

// Weights are held as 2^(z - m + Shift), m the running maximum.  It follows the true one only when logits pass it by far -- a lane's weights of a step add up to more than
// kMostWeight, or a short text's logit passes it by kSlack --, so that most tiles rescale nothing.  f16 ones are lifted by 2^6: their least normal number is
// 2^-14, and small weights of long texts add up.
// z - m is one multiplication and addition where m is small; from kLargePower on the maximum is taken away before the multiplication.
constexpr float kSlack = 8.0f, kMostWeight = 0x1p14f, kMostPower = 0x1.fffffep127f;
template <typename T> struct Shift { static constexpr float value = 0.0f; };
template <> struct Shift<Half> { static constexpr float value = 6.0f; };

template <typename T, int DP, int NW, int RT, int BN, bool DIRECT, bool RUNS>
__global__ __launch_bounds__(NW* kWave, NW == 4 && sizeof(T) == 2 ? 2 : 1) void attention_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * RT * 16, KC = DP / 32, DT = DP / 16;
    constexpr int kPart = RUNS && sizeof(T) == 2 && DP <= 64 ? BN / 16 : 2;            // sixteens of keys whose weights are taken at once
    typedef Tile<T, BN, DP> KeyTile;
    // (variables of their own: reading one does not wait for loads to another)
    __shared__ __align__(16) typename KeyTile::S k_0[KeyTile::kSize], k_1[KeyTile::kSize], v_0[KeyTile::kSize], v_1[KeyTile::kSize];
    typedef typename KeyTile::Place Place;
    const KeyTile k_even{(Place)k_0, (int)threadIdx.x & (kWave - 1)}, k_odd{(Place)k_1, (int)threadIdx.x & (kWave - 1)}, v_even{(Place)v_0, (int)threadIdx.x & (kWave - 1)}, v_odd{(Place)v_1, (int)threadIdx.x & (kWave - 1)};
    extern __shared__ __align__(16) float bias_room[];
    const int W = g.reach + RT * 16 + BN;                      // (a wavefront looks up no places but those of its own tiles)
    const BiasTable table{bias_room, BiasTable::pitch_of(W)};
    int bucket[(2 * (kMaxReach + RT * 16 + BN) + kThreads) / kThreads];
    if (g.bias) BiasTable::look_up<1, kThreads>(g, W, bucket);
    int64_t t;
    int head;
    place_of_workgroup(g, g.heads, t, head);
    const Rows r = rows_of_workgroup<M>(g, t);
    if (!r.mine) return;
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4;
    T* out = static_cast<T*>(g.out) + (int64_t)head * d;
    float* lse = g.lse ? g.lse + (int64_t)head * g.n : nullptr;
    if (r.before || !r.text) {                                 // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0, to = r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span);
        clear_rows(out, g.out_stride, from, to, d);
        for (int64_t i = from + threadIdx.x; lse && i < to; i += kThreads) lse[i] = -__builtin_inff();
        if (!r.text) return;
    }
    const int len = r.len, row0 = r.row0 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * RT * 16;
    const int kv = head / g.group;
    const T* k = static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d;
    const T* v = static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d;

    f32x4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = kLowest;
        l[rt] = 0.0f;
#pragma unroll
        for (int b = 0; b < DT; ++b) o[rt][b] = f32x4{};
    }
    const int steps = r.row0 < len ? (len + BN - 1) / BN : 0;      // (no queries: no keys)
    if (steps) {
        const float cs = g.scale * kLog2e;
        Loader<T, BN, DP, kThreads, DIRECT> next_k(g.k_stride, d), next_v(g.v_stride, d);
        next_k.begin(k_even, k, g.k_stride, 0, len, d);
        next_v.begin(v_even, v, g.v_stride, 0, len, d);
        Fragment<T> q[RT][KC];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int c = 0; c < KC; ++c)
                q[rt][c] = rows_of_memory(static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, row0 + rt * 16, len, d, c, lane);
        if (g.bias) table.fill<kThreads>(g, head, W, min(W, len + M + BN), bucket);
        next_k.finish(k_even);
        next_v.finish(v_even);
        __syncthreads();
        const float before = g.bias ? table.v[0] : 0.0f, behind = g.bias ? table.v[2 * W] : 0.0f;
        auto step = [&](auto kind, int j0, int low, bool near, KeyTile kt, KeyTile vt, KeyTile k_next, KeyTile v_next) __attribute__((always_inline)) {
            constexpr int kKind = decltype(kind)::value;
            if constexpr (kKind != kLast) {
                next_k.begin(k_next, k, g.k_stride, j0 + BN, len, d);
                next_v.begin(v_next, v, g.v_stride, j0 + BN, len, d);
            }
            // what the products are added to: the bias of every place, or of all of them where they are far away
            const float far = low >= g.reach ? behind : before;
            const f32x4 all_far = f32x4{far, far, far, far};
            const float* at = table.from(j0 + quad * 4 - row0 - col + W);
#pragma unroll
            for (int c = 0; c < BN / 16; c += kPart) {
                f32x4 s[RT][kPart];
#pragma unroll
                for (int h = 0; h < kPart; ++h) {
                    if constexpr (kKind != kFar) {
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][h] = kKind == kNear || near ? four_of(at + (c + h - rt) * 16) : all_far;
                    }
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        const Fragment<T> f = kt.rows((c + h) * 16, x);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][h] = multiply(f, q[rt][x], kKind == kFar && x == 0 ? all_far : s[rt][h]);
                    }
                    if constexpr (kKind == kLast) {            // places behind the text's last token
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) s[rt][h][e] = j0 + (c + h) * 16 + quad * 4 + e < len ? s[rt][h][e] : -__builtin_inff();
                    }
                }
                // The weights under the maximum as it is.  Their sum tells whether one of them passes it by far -- sixteen of them are compared at once, which
                // needs no largest one -- and then, seldom, they are taken again.
                Fragment<T> p[RT][kPart / 2];
                float sum[RT];
                auto weigh = [&](auto again) __attribute__((always_inline)) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        // a maximum whose power is large: at first all but -inf weigh infinitely much, and so are taken again
                        const bool large = !(fabsf(m[rt] * cs) < kLargePower);
                        const float off = large ? again.value ? Shift<T>::value : kMostPower : Shift<T>::value - m[rt] * cs, from = again.value && large ? m[rt] : 0.0f;
                        f32x4 sums = f32x4{}, w[kPart];
#pragma unroll
                        for (int h = 0; h < kPart; ++h) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[h][e] = exp2_of(__builtin_fmaf(again.value ? s[rt][h][e] - from : s[rt][h][e], cs, off));
                            sums = sums + w[h];
                        }
                        sum[rt] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
                        for (int h = 0; h < kPart / 2; ++h) p[rt][h] = fragment_of<T>(w[2 * h], w[2 * h + 1]);
                    }
                };
                weigh(std::false_type{});
                bool rises = false;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) rises |= !(sum[rt] <= kMostWeight);
                if (__any(rises)) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        float top = s[rt][0][0];
#pragma unroll
                        for (int h = 0; h < kPart; ++h) top = fmaxf(fmaxf(fmaxf(top, s[rt][h][0]), fmaxf(s[rt][h][1], s[rt][h][2])), s[rt][h][3]);
                        const float now = fmaxf(m[rt], max_of_groups(top)), keep = exp2_of((m[rt] - now) * cs);
                        m[rt] = now;
                        l[rt] *= keep;
#pragma unroll
                        for (int b = 0; b < DT; ++b) o[rt][b] = o[rt][b] * keep;
                    }
                    weigh(std::true_type{});
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) l[rt] += sum[rt];
#pragma unroll
                for (int h = 0; h < kPart / 2; ++h)
#pragma unroll
                    for (int b = 0; b < DT; ++b) {
                        const Fragment<T> f = vt.columns((c + 2 * h) * 16, b);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) o[rt][b] = multiply(f, p[rt][h], o[rt][b]);
                    }
            }
            if constexpr (kKind != kLast) {
                next_k.finish(k_next);
                next_v.finish(v_next);
                __syncthreads();
            }
        };
        walk<RT, BN, RUNS>(g, row0, len, [&](auto kind, auto odd, int i) __attribute__((always_inline)) {
            const int j0 = i * BN, low = j0 - (row0 + RT * 16 - 1), high = j0 + BN - 1 - row0;
            const bool near = g.bias && high > -g.reach && low < g.reach;
            if constexpr (odd.value) step(kind, j0, low, near, k_odd, v_odd, k_even, v_even);
            else step(kind, j0, low, near, k_even, v_even, k_odd, v_odd);
        });
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + rt * 16 + col;
        if (row >= r.span) continue;
        const float sum = sum_of_groups(l[rt]), inverse = row >= len || sum == 0.0f ? 0.0f : 1.0f / sum;
        T* dst = out + (r.begin + row) * g.out_stride;
#pragma unroll
        for (int b = 0; b < DT; ++b) {
            const int c = b * 16 + quad * 4;
            store_piece<T, 4>(dst + c, row < len ? o[rt][b] * inverse : f32x4{}, d - c);
        }
        if (lse && quad == 0)
            lse[r.begin + row] = row >= len || sum == 0.0f ? -__builtin_inff()
                                                           : (m[rt] * (g.scale * kLog2e) + (__builtin_amdgcn_logf(sum) - Shift<T>::value)) * kLn2;
    }
}

// Short texts: a wavefront has 16 queries of several heads, one after the other, and nobody to wait for; keys come straight to registers, values by an LDS
// tile of its own, 32 at a time.  What is the same for all heads -- which text, the distances' buckets where 32 keys are all -- is looked up once.  A workgroup of
// the kernel above has one head of one text, and its chain of look-ups, loads and stores to itself.  4,096 texts of up to 32 tokens, 16 heads of 64 bf16 values:
// 177 us, 3.5 TB/s of the 622 MB that have to move (by the kernel above 433); bound by a wavefront's chain of look-up, loads, two products and store, of which a
// compute unit has sixteen or so at a time.
template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(4 * kWave) void attention_short_kernel(AttentionArgs g, int heads_of_wave) {
    constexpr int M = 16, BN = 32, KC = DP / 32, DT = DP / 16;
    typedef Tile<T, BN, DP> ValueTile;
    __shared__ __align__(16) typename ValueTile::S room[4][ValueTile::kSize];
    typedef typename ValueTile::Place Place;
    const int d = g.d, lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int waves = blockDim.x / kWave, of_workgroup = waves * heads_of_wave;
    const ValueTile vt{(Place)room[wave], lane};
    int64_t t;
    int part;
    place_of_part(g, (g.heads + of_workgroup - 1) / of_workgroup, t, part);
    const Rows r = rows_of_workgroup<M>(g, t);
    if (!r.mine) return;
    const int head0 = part * of_workgroup, head_end = min(g.heads, head0 + of_workgroup);
    if (r.before || !r.text) {                                 // rows of no text
        const int64_t from = r.before ? r.begin - r.before : r.begin + r.row0, to = r.before && r.text ? r.begin : min(r.begin + r.row0 + M, r.begin + r.span);
        clear_rows(static_cast<T*>(g.out) + (int64_t)head0 * d, g.out_stride, from, to, (head_end - head0) * d);
        for (int head = head0; g.lse && head < head_end; ++head)
            for (int64_t i = from + threadIdx.x; i < to; i += blockDim.x) g.lse[(int64_t)head * g.n + i] = -__builtin_inff();
        if (!r.text) return;
    }
    const int len = r.len, row = r.row0 + col;
    const int steps = r.row0 < len ? (len + BN - 1) / BN : 0;
    const float cs = g.scale * kLog2e;
    // places of a lane's eight keys' bias in a head's row, or none
    int bucket[2][4];
    auto look_up = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int b = g.distances[max(-g.reach, min(j0 + h * 16 + quad * 4 + e - row, g.reach)) + g.reach];
                bucket[h][e] = (unsigned)b < (unsigned)g.buckets ? b : -1;
            }
    };
    if (g.bias && steps == 1) look_up(0);
    const uint32_t q_bytes = (uint32_t)g.q_stride * (uint32_t)sizeof(T), k_bytes = (uint32_t)g.k_stride * (uint32_t)sizeof(T);
    Loader<T, BN, DP, kWave, DIRECT> next_v(g.v_stride, d);
    for (int head = head0 + wave; head < head_end; head += waves) {
        const int kv = head / g.group;
        const T* k = static_cast<const T*>(g.k) + r.begin * g.k_stride + (int64_t)kv * d;
        const T* v = static_cast<const T*>(g.v) + r.begin * g.v_stride + (int64_t)kv * d;
        f32x4 o[DT];
        float m = kLowest, l = 0.0f;
#pragma unroll
        for (int b = 0; b < DT; ++b) o[b] = f32x4{};
        Fragment<T> q[KC];
        if (steps) {
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const T* base = static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d;
                if constexpr (DIRECT) q[c] = whole_rows_of_memory(base + r.row0 * g.q_stride, q_bytes, 0, len - 1 - r.row0, d, c, lane);
                else q[c] = rows_of_memory(base, g.q_stride, r.row0, len, d, c, lane);
            }
        }
        for (int j0 = 0; j0 < steps * BN; j0 += BN) {
            next_v.begin(vt, v, g.v_stride, j0, len, d);
            Fragment<T> keys[2][KC];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    if constexpr (DIRECT) keys[h][c] = whole_rows_of_memory(k + j0 * g.k_stride, k_bytes, h * 16, len - 1 - j0, d, c, lane);
                    else keys[h][c] = rows_of_memory(k, g.k_stride, j0 + h * 16, len, d, c, lane);
                }
            f32x4 s[2] = {f32x4{}, f32x4{}};
            if (g.bias) {
                if (steps > 1) look_up(j0);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float entry = scaled_bias(g.bias[(int64_t)head * g.buckets + (uint32_t)max(bucket[h][e], 0)], g.inverse_scale);
                        s[h][e] = bucket[h][e] < 0 ? 0.0f : entry;
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int c = 0; c < KC; ++c) s[h] = multiply(keys[h][c], q[c], s[h]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j0 + h * 16 + quad * 4 + e >= len) s[h][e] = -__builtin_inff();
            }
            const float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            if (__any((top - m) * cs > kSlack)) {
                const float now = fmaxf(m, max_of_groups(top)), keep = exp2_of((m - now) * cs);
                m = now;
                l *= keep;
#pragma unroll
                for (int b = 0; b < DT; ++b) o[b] = o[b] * keep;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[h][e] = exp2_of(__builtin_fmaf(s[h][e] - m, cs, Shift<T>::value));
                    l += s[h][e];
                }
            const Fragment<T> p = fragment_of<T>(s[0], s[1]);
            next_v.finish(vt);
            wave_meets();
#pragma unroll
            for (int b = 0; b < DT; ++b) o[b] = multiply(vt.columns(0, b), p, o[b]);
            wave_meets();
        }
        if (row < r.span) {
            const float sum = sum_of_groups(l), inverse = row >= len || sum == 0.0f ? 0.0f : 1.0f / sum;
            T* dst = static_cast<T*>(g.out) + (r.begin + row) * g.out_stride + (int64_t)head * d;
#pragma unroll
            for (int b = 0; b < DT; ++b) {
                const int c = b * 16 + quad * 4;
                store_piece<T, 4>(dst + c, row < len ? o[b] * inverse : f32x4{}, d - c);
            }
            if (g.lse && quad == 0)
                g.lse[(int64_t)head * g.n + r.begin + row] =
                    row >= len || sum == 0.0f ? -__builtin_inff() : (m * cs + (__builtin_amdgcn_logf(sum) - Shift<T>::value)) * kLn2;
        }
    }
}

}  // namespace

template <typename T>
void launch_attention(const AttentionArgs& args, int rows, bool direct, hipStream_t st) {
    AttentionArgs g = args;
    g.tiles = g.n / rows + g.texts + 1;
    const dim3 blocks((unsigned)(g.tiles * g.heads));
    with_head(g.d, [&](auto dp) {
        constexpr int DP = dp.value, kKeys = sizeof(T) == 4 && DP > 64 ? 32 : 64;
        auto launch = [&](auto kernel, int waves, int most) { hipLaunchKernelGGL(kernel, blocks, dim3(waves * kWave), g.bias ? BiasTable::bytes(most) : 0, st, g); };
        auto of = [&](auto waves, auto rt, auto step, auto runs) {
            constexpr int NW = waves.value, RT = rt.value, BN = step.value;
            if (direct) launch(attention_kernel<T, DP, NW, RT, BN, true, runs.value>, NW, g.reach + RT * 16 + BN);
            else launch(attention_kernel<T, DP, NW, RT, BN, false, false>, NW, g.reach + RT * 16 + BN);
        };
        typedef std::integral_constant<bool, false> No;
        typedef std::integral_constant<bool, true> Yes;
        if (rows == 16) {
            const int waves = std::min(4, g.heads), of_wave = heads_of_a_wavefront(g.tiles, g.heads, waves), parts = (g.heads + waves * of_wave - 1) / (waves * of_wave);
            const dim3 grid((unsigned)(g.tiles * parts)), threads(waves * kWave);
            if (direct && direct_rows(g.q, g.q_stride, sizeof(T), g.d)) hipLaunchKernelGGL((attention_short_kernel<T, DP, true>), grid, threads, 0, st, g, of_wave);
            else hipLaunchKernelGGL((attention_short_kernel<T, DP, false>), grid, threads, 0, st, g, of_wave);
        } else if (rows == 64) of(Width<4>{}, Width<1>{}, Width<kKeys>{}, No{});
        else if (!long_texts(g.n, g.texts)) {
            if constexpr (sizeof(T) == 2 || DP > 96) of(Width<4>{}, Width<2>{}, Width<kKeys>{}, No{});
        } else of(Width<4>{}, Width<2>{}, Width<kKeys>{}, Yes{});
    });
}

}  // namespace pqt
