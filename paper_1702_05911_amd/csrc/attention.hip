// Attention: the C entry, and the usual buckets of distances.
#include <cmath>

#include "attention.hpp"

using pqt_host::DeviceGuard;
using pqt_host::fail;

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
    const int rows = short_texts(n, texts) ? 16 : type == PQT_F32 && few_rows_of_floats(n, texts, d) ? 64 : rows_of_a_workgroup(n, texts, heads);
    with_type(type, [&](auto t) {
        launch_attention<decltype(t)>(g, rows, direct_rows(k, k_stride, sizeof(t), d) && direct_rows(v, v_stride, sizeof(t), d), st);
    });
    HIP_TRY(hipGetLastError());
    return PQT_OK;
}

}  // extern "C"
