// Attention among the tokens of every text: out_i = sum over j of p_ij v_j, p_ij = softmax over j of scale q_i . k_j + bias[bucket of j - i].
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup has 16, 64 or 128 queries of one head, a wavefront one or two times 16
// of them, in registers; tiles of keys and values go through LDS in turn, two of each, the next one on its way from memory.  Products are
// taken transposed -- keys by queries, then values' columns by queries -- so that a lane has one query's logits, and the weights become the second
// product's operand where they are.
#include "attention.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

namespace pqt {
namespace {

// Weights are held as 2^(z - m + kShift), m the running maximum up to 2^kSlack: it follows the true one only when a logit passes it by that much, so that
// most tiles rescale nothing.  f16 ones are lifted by 2^6: their least normal number is 2^-14, and small weights of long texts add up.
constexpr float kSlack = 8.0f;
template <typename T> struct Shift { static constexpr float value = 0.0f; };
template <> struct Shift<Half> { static constexpr float value = 6.0f; };

template <typename T, int DP, int NW, int RT, int BN, bool DIRECT>
__global__ __launch_bounds__(NW* kWave, NW == 4 && sizeof(T) == 2 ? 2 : 1) void attention_kernel(AttentionArgs g) {
    constexpr int kThreads = NW * kWave, M = NW * RT * 16, KC = DP / 32, DT = DP / 16;
    typedef Tile<T, BN, DP> KeyTile;
    // (variables of their own: reading one does not wait for loads to another)
    __shared__ __align__(16) typename KeyTile::S k_0[KeyTile::kSize], k_1[KeyTile::kSize], v_0[KeyTile::kSize], v_1[KeyTile::kSize];
    typedef typename KeyTile::Place Place;
    const KeyTile k_even{(Place)k_0}, k_odd{(Place)k_1}, v_even{(Place)v_0}, v_odd{(Place)v_1};
    extern __shared__ __align__(16) float bias_room[];
    const BiasTable table{bias_room, BiasTable::pitch_of(g.reach + RT * 16 + BN)};
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
        const int W = min(g.reach + RT * 16, len + M) + BN;        // (a wavefront looks up no places but those of its own tiles)
        Loader<T, BN, DP, kThreads, DIRECT> next_k(g.k_stride, d), next_v(g.v_stride, d);
        next_k.begin(k_even, k, g.k_stride, 0, len, d);
        next_v.begin(v_even, v, g.v_stride, 0, len, d);
        if (g.bias) table.fill<1, kThreads>(g, head, W);
        Fragment<T> q[RT][KC];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int c = 0; c < KC; ++c)
                q[rt][c] = rows_of_memory(static_cast<const T*>(g.q) + r.begin * g.q_stride + (int64_t)head * d, g.q_stride, row0 + rt * 16, len, d, c);
        next_k.finish(k_even);
        next_v.finish(v_even);
        __syncthreads();
        const float before = g.bias ? table.v[0] : 0.0f, behind = g.bias ? table.v[2 * W] : 0.0f;
        auto step = [&](int j0, KeyTile kt, KeyTile vt, KeyTile k_next, KeyTile v_next) __attribute__((always_inline)) {
            const bool more = j0 + BN < len;
            if (more) {
                next_k.begin(k_next, k, g.k_stride, j0 + BN, len, d);
                next_v.begin(v_next, v, g.v_stride, j0 + BN, len, d);
            }
            // what the products are added to: the bias of every place, or of all of them where they are far away
            const int low = j0 - (row0 + RT * 16 - 1), high = j0 + BN - 1 - row0;
            const bool near = g.bias && high > -g.reach && low < g.reach;
            const float far = low >= g.reach ? behind : before;
            const float* at = table.from(j0 + quad * 4 - row0 - col + W);
#pragma unroll
            for (int c = 0; c < BN / 32; ++c) {
                f32x4 s[RT][2];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[rt][h] = near ? four_of(at + c * 32 + h * 16 - rt * 16) : f32x4{far, far, far, far};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int x = 0; x < KC; ++x) {
                        const Fragment<T> f = kt.rows(c * 32 + h * 16, x);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) s[rt][h] = multiply(f, q[rt][x], s[rt][h]);
                    }
                if (j0 + c * 32 + 32 > len) {                  // places behind the text's last token
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j0 + c * 32 + h * 16 + quad * 4 + e >= len) {
#pragma unroll
                                for (int rt = 0; rt < RT; ++rt) s[rt][h][e] = -__builtin_inff();
                            }
                }
                float top[RT];
                bool rises = false;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    top[rt] = fmaxf(fmaxf(fmaxf(s[rt][0][0], s[rt][0][1]), fmaxf(s[rt][0][2], s[rt][0][3])), fmaxf(fmaxf(s[rt][1][0], s[rt][1][1]), fmaxf(s[rt][1][2], s[rt][1][3])));
                    rises |= (top[rt] - m[rt]) * cs > kSlack;
                }
                if (__any(rises)) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const float now = fmaxf(m[rt], max_of_groups(top[rt])), keep = exp2_of((m[rt] - now) * cs);
                        m[rt] = now;
                        l[rt] *= keep;
#pragma unroll
                        for (int b = 0; b < DT; ++b) o[rt][b] = o[rt][b] * keep;
                    }
                }
                Fragment<T> p[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float off = Shift<T>::value - m[rt] * cs;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[rt][h][e] = exp2_of(__builtin_fmaf(s[rt][h][e], cs, off));
                            l[rt] += s[rt][h][e];
                        }
                    p[rt] = fragment_of<T>(s[rt][0], s[rt][1]);
                }
#pragma unroll
                for (int b = 0; b < DT; ++b) {
                    const Fragment<T> f = vt.columns(c * 32, b);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) o[rt][b] = multiply(f, p[rt], o[rt][b]);
                }
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

}  // namespace
}  // namespace pqt

extern "C" {

int pqt_distance_buckets(int buckets, int far, int both, int32_t* distances) {
    using namespace pqt;
    if (buckets < 2 || buckets > kMaxBuckets || (both && buckets % 2) || far < 1 || far > kMaxReach || !distances)
        return fail(PQT_EINVAL, "pqt_distance_buckets: buckets=%d (2 to %d, even for both sides), far=%d (1 to %d) or a null pointer", buckets, kMaxBuckets, far, kMaxReach);
    const int side = both ? buckets / 2 : buckets, near = side / 2 > 0 ? side / 2 : 1, rest = side - near;
    if (far < near) return fail(PQT_EINVAL, "pqt_distance_buckets: far=%d is below the %d distances that have a bucket of their own", far, near);
    for (int at = -far; at <= far; ++at) {
        // keys before the query (and it itself) have the first half, those behind it the second; of one-sided buckets these have the first
        const int away = at <= 0 ? -at : both ? at : 0;
        int b = away;
        if (away >= near) {
            b = near;
            // step t begins where log(away / near) / log(far / near) * rest reaches t; 1e-9 above what a logarithm may be short of there
            if (rest > 0 && far > near) b += (int)floor(log((double)away / near) / log((double)far / near) * rest + 1e-9);
        }
        b = std::min(b, side - 1);
        distances[at + far] = b + (both && at > 0 ? side : 0);
    }
    return PQT_OK;
}

int pqt_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int type, int64_t n, int heads,
                  int kv_heads, int d, const void* starts, const void* lengths, int place_bytes, int64_t texts, float scale, const float* bias,
                  int buckets, const int32_t* distances, int reach, int clear, void* out, int64_t out_stride, float* lse, int device,
                  void* hip_stream) {
    using namespace pqt;
    AttentionArgs g{};
    if (const int rc = attention_checks("pqt_attention", type, n, heads, kv_heads, d, starts, lengths, place_bytes, texts, scale, bias, buckets, distances, reach, g)) return rc;
    const int64_t wide = (int64_t)heads * d, narrow = (int64_t)kv_heads * d;
    if (q_stride < wide || k_stride < narrow || v_stride < narrow || out_stride < wide)
        return fail(PQT_EINVAL, "pqt_attention: strides %lld, %lld, %lld, %lld for rows of %lld and %lld values", (long long)q_stride, (long long)k_stride, (long long)v_stride,
                    (long long)out_stride, (long long)wide, (long long)narrow);
    if (n == 0) return PQT_OK;
    if (!q || !k || !v || !out) return fail(PQT_EINVAL, "pqt_attention: null pointer");
    const size_t eb = type_bytes(type);
    if (!aligned_to(q, eb) || !aligned_to(k, eb) || !aligned_to(v, eb) || !aligned_to(out, eb) || !aligned_to(lse, 4))
        return fail(PQT_EINVAL, "pqt_attention: a pointer is not aligned to its element");
    if (const int rc = check_device(device, "pqt_attention")) return rc;
    DeviceGuard guard(device);
    if (!guard.ok) return fail(PQT_EHIP, "cannot select GPU %d", device);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    g.q = q;
    g.k = k;
    g.v = v;
    g.out = out;
    g.lse = lse;
    g.q_stride = q_stride;
    g.k_stride = k_stride;
    g.v_stride = v_stride;
    g.out_stride = out_stride;
    g.clear = clear;
    // (the launch's limits were checked for the smallest workgroups)
    const int rows = rows_of_a_workgroup(n, texts, heads);
    g.tiles = n / rows + texts + 1;
    const unsigned blocks = (unsigned)(g.tiles * heads);
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const bool direct = direct_rows(k, k_stride, sizeof(T), d) && direct_rows(v, v_stride, sizeof(T), d);
        with_head(d, [&](auto dp) {
            constexpr int DP = dp.value, kKeys = sizeof(T) == 4 && DP > 64 ? 32 : 64;
            auto launch = [&](auto kernel, int waves, int most) {
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(waves * kWave), bias ? BiasTable::bytes(most) : 0, st, g);
            };
            auto of = [&](auto waves, auto rt, auto step) {
                constexpr int NW = waves.value, RT = rt.value, BN = step.value;
                if (direct) launch(attention_kernel<T, DP, NW, RT, BN, true>, NW, reach + RT * 16 + BN);
                else launch(attention_kernel<T, DP, NW, RT, BN, false>, NW, reach + RT * 16 + BN);
            };
            if (rows == 16) of(Width<1>{}, Width<1>{}, Width<32>{});
            else if (rows == 64) of(Width<4>{}, Width<1>{}, Width<kKeys>{});
            else of(Width<4>{}, Width<2>{}, Width<kKeys>{});
        });
    });
    HIP_TRY(hipGetLastError());
    return PQT_OK;
}

}  // extern "C"
