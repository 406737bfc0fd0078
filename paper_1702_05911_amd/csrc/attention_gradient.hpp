// What the two kernels of attention's gradients share, and how these are made.  With the weights p_ij = exp(scale q_i . k_j + bias - lse_i) taken again from what the forward pass wrote, delta_i =
// grad_i . out_i and ds_ij = p_ij (grad_i . v_j - delta_i):
//     dq_i = scale sum over j of ds_ij k_j,   dk_j = scale sum over i of ds_ij q_i,   dv_j = sum over i of p_ij grad_i,
//     dbias[head][b] = sum of ds_ij over the distances j - i of bucket b.
//
// Two kernels, so that no sum is anybody else's to add to: one has queries and walks the keys (dq, delta, dbias), one has keys and walks the queries of
// all heads that share them (dk, dv).  Each takes the weights anew, seven products instead of five, and the same inputs give the same bytes.
// Bound by neither unit's rate but by what a step waits for, at two workgroups a compute unit or fewer: 64 texts of up to 512 tokens, 16 heads of 64 bf16 values, 274 us (148 and 138),
// 0.35 PFLOP/s of the seven products; the queries' kernel has the vector unit busy for 44 % of the time and the matrix unit for 16, the keys' for 39 and 23, and their wavefronts wait for 42
// and 37 % of theirs (loads, LDS, barriers).  Two texts of 4,001 and 2,301, 8 heads of 80 f16 values, two of keys, 462 us (244 and 241): 34 and 24 %, 33 and 28, with 0.8 and 1.4
// wavefronts a SIMD of the two that fit, as workgroups do not come out even.
// As in the forward pass the products are turned so that a lane has one own row, whose weights and ds are the next product's operand where they are.
//
// fp32: the keys' kernel takes its weights from lse's rounded power of two, the queries' corrects for it (rest_of_power): 8 texts of up to 48 tokens are 7.2e-7 off, the plain form in 32 bits 5.1e-7.
//
// dbias: a wavefront's ds of 16 queries by 16 keys are added up along their diagonals by moving lanes, so that a lane has one distance, and go to a sum by
// distance in LDS which only this lane's group of sixteen adds to; distances to buckets at the workgroup's end.  Tiles farther away than `reach`
// have one bucket and one sum.
#pragma once
#include "attention.hpp"

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

// From one copy of the sums by distance, -W .. W, to the next: whole pieces of four.
__host__ __device__ constexpr int sums_pitch(int W) { return (2 * W + 4) / 4 * 4; }

// Adds to a number in LDS that nobody else adds to meanwhile.  (LDS' own addition of floats is slow: 64 texts of up to 512 tokens 311 us, 179 so.)
__device__ __forceinline__ void add_to(float* p, float v) { *p += v; }

// A row whose lse is so large that weights cannot be taken from it: with a bias of -1e9 on all that the row has left, the next lse is 64 away.  Such rows have no weights in
// the steps that all rows take.  Where a workgroup meets one, seldom, it walks its text a second time: the queries' kernel takes the row's maximum and sum anew, and both
// take the weights from these.  (This costs others nothing that shows; a question at each of the usual steps instead 2 % on average, up to 10; steps of either kind by
// workgroup 3 %, up to 17, for registers.)
__device__ __forceinline__ bool large_sum(float lse) { return fabsf(lse * kLog2e) >= kLargePower && fabsf(lse) < __builtin_inff(); }
// (Its lanes' places are counted anew, behind a number that the compiler does not see through: shared with the first walk's they would be held in registers all the while.)
struct LaneOf {
    int lane, col, quad;
    __device__ __forceinline__ explicit LaneOf(int l) : lane(l), col(l & 15), quad(l >> 4) {}
    static __device__ __forceinline__ LaneOf anew() {
        int l = threadIdx.x & (kWave - 1);
        asm volatile("" : "+v"(l));
        return LaneOf(l);
    }
};
// (such rows' maxima lie in the room of the second tile then, which that walk has no use for)
typedef float TileFloat __attribute__((may_alias));
typedef f32x4 TileFloats __attribute__((may_alias));

// the logarithm of the sum as a power of two's; rows without weights, and those with a large sum, have none
__device__ __forceinline__ float power_of(float lse) { return fabsf(lse * kLog2e) >= kLargePower ? __builtin_inff() : lse * kLog2e; }
// what weights are to be multiplied by for that power's rounding, the same for all of a row: 1 - rest * ln 2 (the rest is below 2^-12)
__device__ __forceinline__ float rest_of_power(float lse) {
    const float rest = __builtin_fmaf(lse, kLog2e, -(lse * kLog2e)) + lse * kLog2eRest;
    return fabsf(lse * kLog2e) < kLargePower ? __builtin_fmaf(rest, -kLn2, 1.0f) : 1.0f;
}

// Places of the bias table, and of the sums by distance, on either side: those of the tiles that are near, and sixteen for what is carried past one.
template <int RT, int BN>
__host__ __device__ constexpr int most_places(int reach) { return reach + RT * 16 + BN + 16; }

}  // namespace
}  // namespace pqt
