// rs3_rows.cuh -- what the kernels that go over rows share: 16-byte pieces of a row as fp32
// values, and whether two sets of rows share a byte.
#pragma once

#include "rs3_internal.cuh"

template <typename T>
struct Piece;                              // 16 bytes of a row
template <>
struct Piece<uint16_t> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void widen(uint4 v, float *f)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 narrow(const float *f)
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Piece<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void widen(uint4 v, float *f)
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    __device__ static __forceinline__ uint4 narrow(const float *f)
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// Rows of `width` bytes, a_stride and b_stride apart, share no byte: one ends before the other begins, or they are columns
// of the same rows side by side.
inline bool rows_apart(const uint8_t *a, int64_t a_rows, int64_t a_stride, int64_t a_width, const uint8_t *b, int64_t b_rows, int64_t b_stride,
                int64_t b_width)
{
    if (a_rows == 0 || b_rows == 0) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    if (x + (uintptr_t)((a_rows - 1) * a_stride + a_width) <= y || y + (uintptr_t)((b_rows - 1) * b_stride + b_width) <= x) return true;
    if (a_stride != b_stride) return false;
    const uintptr_t n = (uintptr_t)a_stride, off = x >= y ? (x - y) % n : (n - (y - x) % n) % n;      // of a's columns behind b's
    return off >= (uintptr_t)b_width && off + (uintptr_t)a_width <= n;
}
