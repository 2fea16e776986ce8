// 8 adjacent values of a row, at any element's address.
#pragma once
#include "tile_ops.h"

namespace ps {

typedef __attribute__((ext_vector_type(8))) float f32x8_t;
// 16-byte loads from any element's address (element by element, 17776 rows of 1919 bf16 take 44 us)
typedef bf16x8_t any_bf16x8_t __attribute__((aligned(2)));
typedef f32x4_t any_f32x4_t __attribute__((aligned(4)));

// 8 adjacent values of a row of `cols`, from p = the row's value `col` on, zeros behind its end
template <typename T>
__device__ __forceinline__ void load_eight(float (&v)[8], const T* p, int col, int cols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (col + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            const f32x8_t w = __builtin_convertvector(*reinterpret_cast<const any_bf16x8_t*>(p), f32x8_t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = w[i];
        } else {
            const f32x4_t a = *reinterpret_cast<const any_f32x4_t*>(p), c = *reinterpret_cast<const any_f32x4_t*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = c[i]; }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) v[i] = to_f32(p[i]);
    }
}

template <typename T>
__device__ __forceinline__ void store_eight(T* p, const float (&v)[8], int col, int cols) {
    if (col + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<any_bf16x8_t*>(p) = __builtin_convertvector(f32x8_t{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, bf16x8_t);
        } else {
            *reinterpret_cast<any_f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<any_f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) p[i] = from_f32<T>(v[i]);
    }
}

}  // namespace ps
