// What the operators beside the Update stage share (embed.hip, distill.hip, gated.hip): element types, 16-byte pieces of a
// row at any element's address, conversions, argument checks.  Everything lives in the including file's anonymous namespace.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <exception>
#include <string>
#include <type_traits>

#include "plan.hpp"

namespace {

using paro::fail;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

#define PARO_LAUNCHED(what)                                                                              \
    do {                                                                                                 \
        const hipError_t e_ = hipGetLastError();                                                         \
        if (e_ != hipSuccess) return fail(PARO_EHIP, std::string(what ": ") + hipGetErrorString(e_));    \
    } while (0)

// Compile-time loop: the body sees its index as a constant.
template <int I, int N, class F>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// Nothing is thrown across the C boundary: fail() makes strings.
template <class F>
int guarded(F &&f) noexcept {
    try {
        return f();
    } catch (const std::exception &) {
        return PARO_ENOMEM;
    }
}

inline int64_t size_of(int dtype) { return dtype == PARO_F32 ? 4 : 2; }
inline bool is_dtype(int dtype) { return dtype == PARO_BF16 || dtype == PARO_F32 || dtype == PARO_F16; }

// A pointer has to suit its elements; vector loads and stores promise no more.
inline int check_array(const void *p, int64_t size, const std::string &what) {
    if (!p) return fail(PARO_EINVAL, what + " is NULL");
    if (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) return fail(PARO_EALIGN, what + " is not aligned to its elements");
    return PARO_OK;
}
// Whether rows of ld elements reach past 2^62 bytes.
inline bool too_large(int64_t rows, int64_t ld, int64_t size) { return rows > 0 && ld > ((int64_t)1 << 62) / size / rows; }

// ---------------------------------------------------------------- element types
// A piece is 16 bytes: E elements.  It may start at any element (the alignment is part of the pointer's type: one
// instruction all the same).
template <int DT>
struct Elem {
    static constexpr int BYTES = DT == PARO_F32 ? 4 : 2;
    static constexpr int E = 16 / BYTES;
};
typedef u32x4 piece_at2 __attribute__((aligned(2)));
typedef u32x4 piece_at4 __attribute__((aligned(4)));

__device__ __forceinline__ float bits16_to_f32(int dt, unsigned h) {
    return dt == PARO_F16 ? (float)__builtin_bit_cast(_Float16, (unsigned short)h) : __uint_as_float(h << 16);
}
// Round to nearest even; NaN stays NaN.  bf16 pairs go through the hardware's conversion of two.
template <int DT>
__device__ __forceinline__ unsigned f32_to_bits16(float f) {
    if constexpr (DT == PARO_F16) {
        return __builtin_bit_cast(unsigned short, (_Float16)f);
    } else {
        return __builtin_bit_cast(unsigned short, (__bf16)f);
    }
}
template <int DT>
__device__ __forceinline__ unsigned pack2(float a, float b) {
    return f32_to_bits16<DT>(a) | (f32_to_bits16<DT>(b) << 16);
}

template <int DT>
__device__ __forceinline__ void unpack(u32x4 r, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == PARO_F32) {
            x[i] = __uint_as_float(r[i]);
        } else if constexpr (DT == PARO_F16) {
            x[2 * i] = bits16_to_f32(DT, r[i] & 0xFFFFu);
            x[2 * i + 1] = bits16_to_f32(DT, r[i] >> 16);
        } else {
            x[2 * i] = __uint_as_float(r[i] << 16);
            x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        }
    }
}
template <int DT>
__device__ __forceinline__ u32x4 pack(const float *x) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == PARO_F32) r[i] = __float_as_uint(x[i]);
        else r[i] = pack2<DT>(x[2 * i], x[2 * i + 1]);
    }
    return r;
}

template <int DT>
__device__ __forceinline__ u32x4 load_piece(const void *base, int64_t elem) {
    const char *at = static_cast<const char *>(base) + elem * Elem<DT>::BYTES;
    if constexpr (DT == PARO_F32) return *reinterpret_cast<const piece_at4 *>(at);
    else return *reinterpret_cast<const piece_at2 *>(at);
}
template <int DT>
__device__ __forceinline__ void store_piece(void *base, int64_t elem, u32x4 v) {
    char *at = static_cast<char *>(base) + elem * Elem<DT>::BYTES;
    if constexpr (DT == PARO_F32) *reinterpret_cast<piece_at4 *>(at) = v;
    else *reinterpret_cast<piece_at2 *>(at) = v;
}
// ... of what is touched once and larger than the caches.
template <int DT>
__device__ __forceinline__ u32x4 load_stream(const void *base, int64_t elem) {
    const char *at = static_cast<const char *>(base) + elem * Elem<DT>::BYTES;
    if constexpr (DT == PARO_F32) return __builtin_nontemporal_load(reinterpret_cast<const piece_at4 *>(at));
    else return __builtin_nontemporal_load(reinterpret_cast<const piece_at2 *>(at));
}
template <int DT>
__device__ __forceinline__ void store_stream(void *base, int64_t elem, u32x4 v) {
    char *at = static_cast<char *>(base) + elem * Elem<DT>::BYTES;
    if constexpr (DT == PARO_F32) __builtin_nontemporal_store(v, reinterpret_cast<piece_at4 *>(at));
    else __builtin_nontemporal_store(v, reinterpret_cast<piece_at2 *>(at));
}
// Four elements of a two-byte type.
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 half_piece_at2 __attribute__((aligned(2)));
__device__ __forceinline__ u32x2 load_half_piece_stream(const void *base, int64_t elem) {
    return __builtin_nontemporal_load(reinterpret_cast<const half_piece_at2 *>(static_cast<const char *>(base) + elem * 2));
}
__device__ __forceinline__ u32x2 load_half_piece(const void *base, int64_t elem) {
    return *reinterpret_cast<const half_piece_at2 *>(static_cast<const char *>(base) + elem * 2);
}
__device__ __forceinline__ void store_half_piece(void *base, int64_t elem, u32x2 v) {
    *reinterpret_cast<half_piece_at2 *>(static_cast<char *>(base) + elem * 2) = v;
}
template <int DT>
__device__ __forceinline__ float load_one(const void *base, int64_t elem) {
    if constexpr (DT == PARO_F32) return static_cast<const float *>(base)[elem];
    else return bits16_to_f32(DT, static_cast<const unsigned short *>(base)[elem]);
}
template <int DT>
__device__ __forceinline__ void store_one(void *base, int64_t elem, float v) {
    if constexpr (DT == PARO_F32) static_cast<float *>(base)[elem] = v;
    else static_cast<unsigned short *>(base)[elem] = (unsigned short)f32_to_bits16<DT>(v);
}

}  // namespace
