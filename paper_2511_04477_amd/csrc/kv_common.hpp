// Device code that the kernels of the key/value cache share (spqt_kv.h has the layout and the quantization rule).
#ifndef SPQT_KV_COMMON_HPP
#define SPQT_KV_COMMON_HPP

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "spqt_internal.h"
#include "spqt_kv.h"

namespace spqt {
namespace kv {

constexpr int kBlock = SPQT_KV_BLOCK;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// What a kernel knows of a cache: spqt_kv_cache without what it does not use.
struct Cache {
    uint8_t *codes;
    float *scales;
    uint16_t *tail;
    float *weights;
    const int32_t *table;
    const int32_t *lengths;
    uint32_t pages;
    int max_blocks, kv_heads, head_dim;
};
struct Rows {
    uint16_t *data;
    int64_t sequence, row, head;
};

// Where a token lies in the 64 bytes of one element of the values: the order in which a lane of the matrix instructions wants them.
__host__ __device__ inline int place_of(int t) { return 16 * (t / 4 % 4) + 4 * (t / 16) + t % 4; }

__device__ __forceinline__ float as_float(uint32_t bits) { return __builtin_bit_cast(float, bits); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }

template <bool BF16>
__device__ __forceinline__ float widen(uint16_t x) {
    return BF16 ? as_float((uint32_t)x << 16) : (float)__builtin_bit_cast(_Float16, x);
}
// Two numbers to nearest even, the first one in the lower half.
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}

// The scale of a block whose largest |x| this is.
__device__ __forceinline__ float scale_for(float largest) {
    float t = largest / 127.0f;
    t = t > 0x1p-100f ? t : 0x1p-100f;
    const uint32_t bits = as_u32(t);
    uint32_t odd = (bits & ~0x1FFFu) | 0x1000u;
    if (odd < bits) odd += 0x2000u;
    return as_float(odd);
}
// The same from the 16 bits of the largest |x| (NaN and infinities order above all numbers, and give NaN).
template <bool BF16>
__device__ __forceinline__ float scale_of(uint32_t largest) {
    return largest >= (BF16 ? 0x7F80u : 0x7C00u) ? __builtin_nanf("") : scale_for(widen<BF16>((uint16_t)largest));
}

// The stored byte of x in the lowest bits of a number, given 1 / scale: adding 1.5 2^23 rounds to the nearest integer.  x * inverse is x / scale to 2^-24 of
// itself, and x / scale is at least 2^-20 of itself away from the middle between two integers, so it rounds as the quotient does.
__device__ __forceinline__ uint32_t coded(float x, float inverse) { return as_u32(__builtin_fmaf(x, inverse, 12582912.0f + 128.0f)); }
// Four of them; what is no number, in a block whose scale is none, is stored as 0.
__device__ __forceinline__ uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {
    const uint32_t low = __builtin_amdgcn_perm(b, a, 0x0C0C0400u), high = __builtin_amdgcn_perm(d, c, 0x04000C0Cu);
    return scale != scale ? 0x80808080u : low | high;
}

// The same for numbers that are finite or NaN and at most 127 times a scale: the type's largest number where they round to infinity.  127 scale_of(65504) = 65563.75 does; a bf16 never,
// since 127 scale is less than 2^-10 above the largest |x| and the largest bf16 number 2^-9 below where rounding leaves the type.
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2_within(float a, float b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const uint32_t x = narrow2<BF16>(a, b);
    if (BF16) return x;
    const u16x2 finite = __builtin_elementwise_min(__builtin_bit_cast(u16x2, (x & 0x7FFF7FFFu) ^ 0x7C007C00u), u16x2{1, 1});     // 0 for an infinity
    return __builtin_bit_cast(uint32_t, (u16x2)(__builtin_bit_cast(u16x2, x) + finite - u16x2{1, 1}));
}

// Two cached values as a reader gets them.
template <bool BF16>
__device__ __forceinline__ uint32_t values_of(uint32_t first, uint32_t second, float scale) {
    const float largest = BF16 ? as_float(0x7F7F0000u) : 65504.0f;
    auto value = [&](uint32_t byte) {
        const float v = (float)((int)byte - 128) * scale;
        return v != v ? v : __builtin_fmaxf(-largest, __builtin_fminf(v, largest));
    };
    return narrow2<BF16>(value(first), value(second));
}

__device__ __forceinline__ int clamped(int v, int low, int high) { return v < low ? low : (v > high ? high : v); }
__device__ __forceinline__ int length_of(const Cache &c, int s) { return clamped(c.lengths[s], 0, c.max_blocks * kBlock); }
__device__ __forceinline__ int count_of(const int32_t *counts, int s, int rows) { return counts ? clamped(counts[s], 0, rows) : rows; }
__device__ __forceinline__ int block_of(int position) { return position >> 6; }       // of a negative one too

// First byte of the keys (0) or values (1) of a page and head.
__device__ __forceinline__ size_t codes_at(const Cache &c, uint32_t page, int head, int which) {
    return (((size_t)page * (size_t)c.kv_heads + (size_t)head) * 2 + (size_t)which) * (size_t)(kBlock * c.head_dim);
}
__device__ __forceinline__ size_t scale_at(const Cache &c, uint32_t page, int head, int which) {
    return ((size_t)page * (size_t)c.kv_heads + (size_t)head) * 2 + (size_t)which;
}
__device__ __forceinline__ size_t weight_at(const Cache &c, uint32_t page, int head) {
    return ((size_t)page * (size_t)c.kv_heads + (size_t)head) * kBlock;
}

// Lane l's value of lanes 0 .. l together; lane 63 has all.
template <class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));      // row_shr:1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));      // row_bcast:15
    return f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));   // row_bcast:31
}
__device__ __forceinline__ uint32_t sum_upto(uint32_t v) {
    return over_lanes(v, [](uint32_t x, uint32_t y) { return x + y; });
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }

// Eight stored bytes as the fp16 numbers code (exact).
__device__ __forceinline__ f16x8 codes_f16(u32x2 w) {
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};      // 1024, which the bytes are put over, and 128
    union {
        f16x2 part[4];
        f16x8 all;
    } r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r.part[2 * i] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w[i], 0x04010400u)) - bias;
        r.part[2 * i + 1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w[i], 0x04030402u)) - bias;
    }
    return r.all;
}

// ---- host

inline int check_cache(const spqt_kv_cache *c, bool tail) {
    if (!c || !c->codes || !c->scales || !c->table || !c->lengths || (tail && !c->tail)) return SPQT_EINVAL;
    if (c->type != SPQT_KV_FP16 && c->type != SPQT_KV_BF16) return SPQT_EINVAL;
    if (c->pages < 1 || c->pages > 0x7FFFFFFF || c->sequences < 1 || c->sequences > 65535) return SPQT_ESHAPE;
    if (c->max_blocks < 1 || c->max_blocks > 1 << 24 || c->kv_heads < 1 || c->kv_heads > 16384) return SPQT_ESHAPE;
    if (c->head_dim < 64 || c->head_dim > SPQT_KV_MAX_DIM || c->head_dim % 64 != 0) return SPQT_ESHAPE;
    if ((uintptr_t)c->codes % 16 != 0 || (uintptr_t)c->scales % 8 != 0 || (uintptr_t)c->tail % 16 != 0 || (uintptr_t)c->weights % 16 != 0 ||
        (uintptr_t)c->table % 4 != 0 || (uintptr_t)c->lengths % 4 != 0)
        return SPQT_EALIGN;
    return SPQT_OK;
}
inline int check_rows(const spqt_kv_rows *r) {
    if (!r || !r->data) return SPQT_EINVAL;
    if (r->sequence < 0 || r->row < 0 || r->head < 0) return SPQT_EINVAL;
    if ((uintptr_t)r->data % 16 != 0 || r->sequence % 8 != 0 || r->row % 8 != 0 || r->head % 8 != 0) return SPQT_EALIGN;
    return SPQT_OK;
}
constexpr int kMaxRows = 1 << 21;

inline Cache view(const spqt_kv_cache &c) {
    return {(uint8_t *)c.codes, c.scales, (uint16_t *)c.tail, c.weights, c.table, c.lengths, (uint32_t)c.pages, c.max_blocks, c.kv_heads, c.head_dim};
}
inline Rows view(const spqt_kv_rows &r) { return {(uint16_t *)r.data, r.sequence, r.row, r.head}; }

// f(constant head_dim, constant BF16) for the cache's.
template <class F>
inline void dispatch(const spqt_kv_cache &c, F f) {
    auto typed = [&](auto dim) {
        if (c.type == SPQT_KV_BF16) f(dim, std::true_type());
        else f(dim, std::false_type());
    };
    switch (c.head_dim) {
        case 64: typed(std::integral_constant<int, 64>()); break;
        case 128: typed(std::integral_constant<int, 128>()); break;
        case 192: typed(std::integral_constant<int, 192>()); break;
        default: typed(std::integral_constant<int, 256>()); break;
    }
}
inline int launched() { return hipGetLastError() == hipSuccess ? SPQT_OK : SPQT_EHIP; }

}  // namespace kv
}  // namespace spqt
#endif
