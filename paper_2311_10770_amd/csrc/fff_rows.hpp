// fff_rows.hpp -- loads and stores of row elements whose type is a run-time value
// and whose rows start at any element.
#pragma once

#include "fff_device.hpp"

#include <hip/hip_runtime.h>

#include <cstdint>

namespace fff {

// Two values rounded to bf16 by one instruction (pack_bf16x2's separate roundings take four).
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, bf16x2_t));
}

__device__ __forceinline__ float load_elem(const void* p, bool bf, int64_t i) {
    return bf ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_elem(void* p, bool bf, int64_t i, float v) {
    if (bf) static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// Four values of a row as they lie in memory, from element e on, `left` of
// them in the row (zeros behind it).  Rows start wherever the row length puts them: global accesses
// of 8 and 16 bytes need no alignment of their own.
typedef uint32_t Raw4 __attribute__((ext_vector_type(4)));  // bf16: two words
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

template <bool FULL>
__device__ __forceinline__ Raw4 load4(const void* base, int bf, int64_t e, int left) {
    Raw4 r = {0, 0, 0, 0};
    if (bf) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + e;
        if (FULL || left >= 4) {
            const u32x2_a2 v = *reinterpret_cast<const u32x2_a2*>(p);
            r.x = v.x;
            r.y = v.y;
        } else {
            if (left > 0) r.x = p[0];
            if (left > 1) r.x |= uint32_t(p[1]) << 16;
            if (left > 2) r.y = p[2];
        }
    } else {
        const uint32_t* p = static_cast<const uint32_t*>(base) + e;
        if (FULL || left >= 4) {
            r = *reinterpret_cast<const u32x4_a4*>(p);
        } else {
            if (left > 0) r.x = p[0];
            if (left > 1) r.y = p[1];
            if (left > 2) r.z = p[2];
        }
    }
    return r;
}
__device__ __forceinline__ void unpack4(float* f, const Raw4& r, int bf) {
    f[0] = __uint_as_float(bf ? r.x << 16 : r.x);
    f[1] = __uint_as_float(bf ? r.x & 0xffff0000u : r.y);
    f[2] = __uint_as_float(bf ? r.y << 16 : r.z);
    f[3] = __uint_as_float(bf ? r.y & 0xffff0000u : r.w);
}
template <bool FULL>
__device__ __forceinline__ void store4(void* base, int bf, int64_t e, int left, const float* f) {
    if (bf) {
        uint16_t* p = static_cast<uint16_t*>(base) + e;
        if (FULL || left >= 4) {
            *reinterpret_cast<u32x2_a2*>(p) = u32x2_a2{pack2(f[0], f[1]), pack2(f[2], f[3])};
        } else {
            if (left > 0) p[0] = f32_to_bf16(f[0]);
            if (left > 1) p[1] = f32_to_bf16(f[1]);
            if (left > 2) p[2] = f32_to_bf16(f[2]);
        }
    } else {
        float* p = static_cast<float*>(base) + e;
        if (FULL || left >= 4) {
            *reinterpret_cast<u32x4_a4*>(p) = u32x4_a4{__float_as_uint(f[0]), __float_as_uint(f[1]),
                                                       __float_as_uint(f[2]), __float_as_uint(f[3])};
        } else {
            if (left > 0) p[0] = f[0];
            if (left > 1) p[1] = f[1];
            if (left > 2) p[2] = f[2];
        }
    }
}

// Eight values from element e on of a matrix of `all` elements: bf16 in one 16-byte load, fp32 in two.
// A vector may run on into the next row (its values are the caller's to leave out): only those that
// end behind the matrix are read one by one, so that no row's tail costs eight loads.  WHOLE: none does.
struct Raw8 {
    Raw4 a, b;  // bf16: a alone
};
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));

template <bool WHOLE = false>
__device__ __forceinline__ Raw8 load8(const void* base, int bf, int64_t e, int64_t all) {
    Raw8 r = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (bf) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + e;
        if (WHOLE || e + 8 <= all) {
            r.a = *reinterpret_cast<const u32x4_a2*>(p);
        } else {
            for (int j = 0; j < 8 && e + j < all; ++j) r.a[j / 2] |= uint32_t(p[j]) << (j % 2 * 16);
        }
    } else {
        const uint32_t* p = static_cast<const uint32_t*>(base) + e;
        if (WHOLE || e + 8 <= all) {
            r.a = *reinterpret_cast<const u32x4_a4*>(p);
            r.b = *reinterpret_cast<const u32x4_a4*>(p + 4);
        } else {
            for (int j = 0; j < 8 && e + j < all; ++j) (j < 4 ? r.a : r.b)[j % 4] = p[j];
        }
    }
    return r;
}
__device__ __forceinline__ void unpack8(float* f, const Raw8& r, int bf) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(bf ? r.a[j] << 16 : j < 2 ? r.a[2 * j] : r.b[2 * j - 4]);
        f[2 * j + 1] = __uint_as_float(bf ? r.a[j] & 0xffff0000u : j < 2 ? r.a[2 * j + 1] : r.b[2 * j - 3]);
    }
}
// `left` of the eight are in the row.
__device__ __forceinline__ void store8(void* base, int bf, int64_t e, int left, const float* f) {
    if (left >= 8) {
        if (bf) {
            *reinterpret_cast<u32x4_a2*>(static_cast<uint16_t*>(base) + e) =
                u32x4_a2{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])};
        } else {
            store4<true>(base, 0, e, 4, f);
            store4<true>(base, 0, e + 4, 4, f + 4);
        }
    } else {
        store4<false>(base, bf, e, left, f);
        if (left > 4) store4<false>(base, bf, e + 4, left - 4, f + 4);
    }
}

}  // namespace fff
