// Matrix instructions of gfx950 and the layouts that the operators build on.
//
// v_mfma_f32_32x32x16: D[m][n] += sum_k A[m][k] B[k][n].  Lane l = 32 h + i holds A[i][8 h + j] and B[8 h + j][i] for j = 0 .. 7,
// and D[8 (r / 4) + 4 h + r % 4][i] for r = 0 .. 15.  The sixteen values of a lane are one column of D: with keys along m
// and query rows along n a lane holds scores of one row only, and eight consecutive values are, rounded, the B operand of a
// second product whose summation index runs over m in the order 4 h + {0 .. 3}, 8 + 4 h + {0 .. 3}.  Its A operand comes
// from row-major memory by two transposing reads (ds_read_b64_tr_b16): sixteen lanes read four rows of sixteen
// 16-bit values, eight bytes a lane, and lane i receives the four values of column i.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace mmee {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct F16 {
    typedef _Float16 Scalar;
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    typedef _Float16 V4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mma(V8 a, V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

struct BF16 {
    typedef __bf16 Scalar;
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    typedef __bf16 V4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mma(V8 a, V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// Types whose normal numbers end well above the smallest probabilities and gradients.
template <class T>
constexpr bool NARROW = std::is_same_v<T, F16>;

// A row-major tile of 16-bit values in shared memory, CH chunks of eight values a row.  Chunk c of row r lies at place
// c ^ spread(r): 16 rows' reads of one chunk (A and B operands along the rows) then meet every bank once, and so do four
// rows' reads of 64 neighbouring bytes (the transposing reads).
template <int CH>
__device__ __forceinline__ int spread(int row)
{
    static_assert(CH >= 4 && CH <= 32 && (CH & (CH - 1)) == 0, "rows of 64 to 512 bytes");
    constexpr int W = CH > 16 ? 16 : CH;                // chunks within the 256 bytes that the banks span
    const int q = row / (16 / W);
    return ((q & (W / 4 - 1)) << 2) | ((q / (W / 4)) & 3);
}

template <int CH>
__device__ __forceinline__ int chunk_at(int row, int c) { return row * CH + (c ^ spread<CH>(row)); }

// Four values of a column: rows `row` .. +3 of the addresses that its sixteen lanes give.
__device__ __forceinline__ s16x4 read_transposed(const void *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}

// A buffer of 2^31 bytes from a pointer on: more than a tile spans.  Loads at BEYOND give zeros.
constexpr uint32_t BEYOND = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const uint16_t *p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p), 0, (int)BEYOND, 0x00027000); }

// Shared memory that only one wave uses: its accesses stay in order.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <class T>
__device__ __forceinline__ typename T::V8 join(s16x4 lo, s16x4 hi)
{
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(typename T::V8, both);
}

template <class T>
__device__ __forceinline__ typename T::V8 as_operand(u32x4 v) { return __builtin_bit_cast(typename T::V8, v); }

// Maximum and sum over the lanes l and l ^ 32.
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace mmee
