// What the kernels of spqt_i8.h share.
#ifndef SPQT_I8_COMMON_HPP
#define SPQT_I8_COMMON_HPP

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "spqt_i8.h"
#include "spqt_internal.h"

namespace spqt {
namespace i8 {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
// Vectors at any element: the memory takes 16 bytes of a lane at any address.
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));

__device__ __forceinline__ float as_float(uint32_t bits) { return __builtin_bit_cast(float, bits); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }

template <bool BF16>
__device__ __forceinline__ float widen(uint32_t x) {
    return BF16 ? as_float(x << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)x);
}
// Two numbers to nearest even, the first one in the lower half.
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}

// ---- host

inline int launched() { return hipGetLastError() == hipSuccess ? SPQT_OK : SPQT_EHIP; }
inline bool sixteen_bits(int type) { return type == SPQT_I8_FP16 || type == SPQT_I8_BF16; }

// [rows][K] with this stride, of elements of `bytes`; written: rows must not overlap.
inline int check_matrix(const void *data, int64_t stride, int64_t rows, int64_t K, int bytes, bool written) {
    if (!data || stride < 0 || (written && rows > 1 && stride < K)) return SPQT_EINVAL;
    if (stride > (int64_t)1 << 40) return SPQT_ESHAPE;
    return (uintptr_t)data % bytes != 0 ? SPQT_EALIGN : SPQT_OK;
}
inline int check_codes(const void *data, int64_t stride, int64_t rows, int64_t K, bool written) {
    const int rc = check_matrix(data, stride, rows, K, 16, written);
    if (rc != SPQT_OK) return rc;
    return stride % 16 != 0 ? SPQT_EALIGN : SPQT_OK;
}
inline int check_extents(int64_t rows, int64_t K, int64_t most) {
    return rows < 1 || rows > SPQT_I8_MAX_ROWS || K < 1 || K > most ? SPQT_ESHAPE : SPQT_OK;
}
inline int check_scales(const float *s) { return !s ? SPQT_EINVAL : (uintptr_t)s % 4 != 0 ? SPQT_EALIGN : SPQT_OK; }

}  // namespace i8
}  // namespace spqt
#endif
