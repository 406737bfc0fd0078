// What the query encoder's kernels share (embed.hip, layer_norm.hip, block_quantize.hip, block_product.hip): the element
// types, rows read and written in pieces, sums over a group of lanes, and the checks of the C entries.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pqt_device.hpp"
#include "pqt_index.hpp"

namespace pqt {

struct Bf16 { uint16_t bits; };
typedef _Float16 Half;

// Pieces of a row.  Rows begin wherever an element may (odd lengths, slices of wider buffers): the pieces are declared
// with the alignment of one element, and the memory system takes 16-byte accesses at such addresses as they are.
template <typename T> struct Vec;
template <> struct Vec<float> {
    typedef float v4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef float v8 __attribute__((ext_vector_type(8), aligned(4)));
};
template <> struct Vec<Bf16> {
    typedef __bf16 v4 __attribute__((ext_vector_type(4), aligned(2)));
    typedef __bf16 v8 __attribute__((ext_vector_type(8), aligned(2)));
};
template <> struct Vec<Half> {
    typedef _Float16 v4 __attribute__((ext_vector_type(4), aligned(2)));
    typedef _Float16 v8 __attribute__((ext_vector_type(8), aligned(2)));
};
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <int N> struct Floats;
template <> struct Floats<4> { typedef f32x4 type; };
template <> struct Floats<8> { typedef f32x8 type; };
template <typename T> struct Element { typedef T type; };
template <> struct Element<Bf16> { typedef __bf16 type; };
template <typename T, int N> struct Piece_;
template <typename T> struct Piece_<T, 4> { typedef typename Vec<T>::v4 type; typedef typename Element<T>::type element; };
template <typename T> struct Piece_<T, 8> { typedef typename Vec<T>::v8 type; typedef typename Element<T>::type element; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(Half v) { return (float)v; }
__device__ __forceinline__ float to_float(Bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
template <typename T> __device__ __forceinline__ T from_float(float v);           // to nearest even
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ Half from_float<Half>(float v) { return (Half)v; }
template <> __device__ __forceinline__ Bf16 from_float<Bf16>(float v) { return Bf16{__builtin_bit_cast(uint16_t, (__bf16)v)}; }

// N elements at p as they are; `have` of them exist (the rest are zeros, not read from memory)
template <typename T, int N>
__device__ __forceinline__ typename Piece_<T, N>::type load_raw(const T* p, int have) {
    typedef typename Piece_<T, N>::type V;
    if (have >= N) return *reinterpret_cast<const V*>(p);
    V out = {};
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < have) out[j] = __builtin_bit_cast(typename Piece_<T, N>::element, p[j]);
    return out;
}

// N elements at p as floats; `have` of them exist (the rest are read as zeros, not at all from memory)
template <typename T, int N>
__device__ __forceinline__ typename Floats<N>::type load_piece(const T* p, int have) {
    typedef typename Floats<N>::type F;
    if (have >= N) return __builtin_convertvector(*reinterpret_cast<const typename Piece_<T, N>::type*>(p), F);
    F out;
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = j < have ? to_float(p[j]) : 0.0f;
    return out;
}

// Results of more bytes than the eight XCDs' L2 hold are stored past it by lookups, layer norm and the wide products, so that they do not push out what is still
// to be read, nor are written back in the next kernel's time (a lookup of 100,003 x 1,024 floats takes 82 us so and 122 otherwise; calls of
// layer norm over 65,537 x 960 follow each other in 48.8 us and in 53.3, though one alone takes 49 and 46; cutting and product of
// 16,384 x 4,096 x 4,096 in 263 and 266); smaller ones stay for
// whoever reads them next.  (Not the layer norm's gradient, which reads twice what it writes: 16,384 x 4,096 80 us a call either way.)
constexpr double kStreamBytes = 32.0 * (1 << 20);
template <typename V>
__device__ __forceinline__ void store_vector(V* p, V v, bool stream) {
    if (stream) {                              // (the empty statements keep the compiler from making one ordinary store of both)
        asm volatile("");
        __builtin_nontemporal_store(v, p);
        asm volatile("");
    } else *p = v;
}

template <typename T, int N>
__device__ __forceinline__ void store_piece(T* p, typename Floats<N>::type v, int have, bool stream = false) {
    typedef typename Piece_<T, N>::type V;
    if (have >= N) {
        store_vector(reinterpret_cast<V*>(p), __builtin_convertvector(v, V), stream);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < have) p[j] = from_float<T>(v[j]);
}

// The piece of N values that a lane reads of a row of D >= N where its own values begin at c: the last piece begins earlier, so that it is
// whole and no lane takes another path; values before `own` are a neighbour's too, and are not stored.
template <int N>
struct WholePiece {
    int64_t c;
    int own;
    __device__ __forceinline__ WholePiece(int64_t from, int64_t D) : c(from < D - N ? from : D - N), own((int)min(from - c, (int64_t)N)) {}
    template <typename T>
    __device__ __forceinline__ typename Piece_<T, N>::type load(const T* row) const {
        return *reinterpret_cast<const typename Piece_<T, N>::type*>(row + c);
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, typename Floats<N>::type v, bool stream) const {
        typedef typename Piece_<T, N>::type V;
        if (own == 0) {
            store_vector(reinterpret_cast<V*>(row + c), __builtin_convertvector(v, V), stream);
            return;
        }
#pragma unroll
        for (int j = 1; j < N; ++j)
            if (j >= own) row[c + j] = from_float<T>(v[j]);
    }
};

// Sum over the G lanes of a group (G a power of two up to 64, groups aligned), in every lane; the order of the additions is
// fixed.
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    if constexpr (G >= 2) v += dpp_move<0xB1>(v);                        // lane ^ 1
    if constexpr (G >= 4) v += dpp_move<0x4E>(v);                        // lane ^ 2
    if constexpr (G >= 8) v += dpp_move<0x141>(v);                       // the other four of eight lanes
    if constexpr (G >= 16) v += dpp_move<0x140>(v);                      // the other eight of sixteen
    if constexpr (G >= 32) v += __uint_as_float((uint32_t)__builtin_amdgcn_ds_swizzle((int)__float_as_uint(v), (16 << 10) | 0x1f));
    if constexpr (G >= 64) v += __shfl_xor(v, 32, kWave);
    return v;
}

// ---- checks of the C entries -----------------------------------------------------------------------------------------
inline bool known_type(int type) { return type == PQT_F32 || type == PQT_BF16 || type == PQT_F16; }
inline size_t type_bytes(int type) { return type == PQT_F32 ? 4 : 2; }
// (nullptr, and pointers off their element's alignment, are refused: a kernel would read or write at half an element)
inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

inline int check_device(int device, const char* who) {
    static const int ndev = [] {                               // (it does not change while a process runs)
        int n = 0;
        if (hipGetDeviceCount(&n) != hipSuccess) {
            (void)hipGetLastError();
            n = 0;
        }
        return n;
    }();
    if (device < 0 || device >= ndev) return pqt_host::fail(PQT_EHIP, "%s: GPU %d is not available (%d visible)", who, device, ndev);
    return PQT_OK;
}

// calls f(T{}) with the element type that `type` names
template <typename F>
inline void with_type(int type, F&& f) {
    if (type == PQT_F32) f(float{});
    else if (type == PQT_BF16) f(Bf16{});
    else f(Half{});
}

}  // namespace pqt
