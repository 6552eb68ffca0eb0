// Matrix-core fragments of the operators.  Internal to a translation unit (anonymous namespace).
//
// One product D[m][n] += sum_k A[m][k] B[k][n] is 32 x 32 with 16 steps of k, for both types: lane l holds eight k of row
// (A) or column (B) l % 32, namely k = 8 h + 0..7 with h = l / 32.  bf16 is one v_mfma_f32_32x32x16_bf16; f32 is eight
// v_mfma_f32_32x32x2_f32, the j-th of which takes element j of both halves.  The numbering of k is free as long as A and
// B agree on it.  D: lane l holds column l % 32, register r row (r % 4) + 8 (r / 4) + 4 h.
// So the registers 8c .. 8c+7 of a D are, converted, the fragment of a next product whose k runs over the rows of D: element j
// of chunk c is row 16 c + 8 (j / 4) + 4 h + j % 4 (`frag_of`).  load_t reads the other operand in that numbering.
#ifndef KT_MFMA_H
#define KT_MFMA_H

#include "kt_ops_device.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define KT_LDS __attribute__((address_space(3)))

namespace {

template <typename T> struct Frag;
template <> struct Frag<bf16> { typedef bf16x8 type; };
template <> struct Frag<float> { typedef f32x8 type; };

__device__ __forceinline__ void mma(f32x16 &d, bf16x8 a, bf16x8 b)
{
    d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16 &d, f32x8 a, f32x8 b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], d, 0, 0, 0);
}

// Chunk c (0 or 1) of a D as a fragment over its rows; bf16: rounded to nearest-even.
template <typename T> __device__ __forceinline__ typename Frag<T>::type frag_of(const f32x16 &d, int c);
template <> __device__ __forceinline__ bf16x8 frag_of<bf16>(const f32x16 &d, int c)
{
    f32x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = d[8 * c + j];
    return __builtin_convertvector(v, bf16x8);
}
template <> __device__ __forceinline__ f32x8 frag_of<float>(const f32x16 &d, int c)
{
    f32x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = d[8 * c + j];
    return v;
}

// Tiles in LDS: rows of W elements (a power of two), their 16-byte chunks exchanged within a row so that both ways of reading
// them spread over all banks (64 banks of 4 bytes):
//   along rows (load_r), 16 lanes read the same chunk of 16 rows that follow each other;
//   across rows (load_t), 32 lanes read 64 adjacent bytes of 4 rows that follow each other.
// Rows of 256 bytes and more: chunk ^ ((row % 4) * 4 + row / 4 % 4) puts 4 rows into the 4 quarters of 256 bytes, and 16
// rows into 16 different chunks.  Rows of 128 bytes: two rows fill the banks; chunk ^ (row / 2 % 2 * 4 + row / 4 % 4).
template <typename T, int W> struct Tile {
    static constexpr int CHUNKS = W * (int)sizeof(T) / 16;
    static_assert(CHUNKS >= 8 && (CHUNKS & (CHUNKS - 1)) == 0, "rows of 128 bytes at least");
    static constexpr int bytes(int rows) { return rows * W * (int)sizeof(T); }
    static __device__ __forceinline__ int swizzle(int row)
    {
        return CHUNKS >= 16 ? (row & 3) * 4 + (row >> 2 & 3) : (row >> 1 & 1) * 4 + (row >> 2 & 3);
    }
    // byte offset of a row's chunk
    static __device__ __forceinline__ int at(int row, int chunk) { return (row * CHUNKS + (chunk ^ swizzle(row))) * 16; }
};

// Fragment along rows: eight elements of row `row0 + lane % 32` from column 16 c + 8 h on.
template <typename T, int W>
__device__ __forceinline__ typename Frag<T>::type load_r(const char *tile, int row0, int c)
{
    const int l = threadIdx.x & 63, row = row0 + (l & 31), h = l >> 5;
    if constexpr (sizeof(T) == 2) {
        return *(const bf16x8 *)(tile + Tile<T, W>::at(row, 2 * c + h));
    } else {
        const f32x4 lo = *(const f32x4 *)(tile + Tile<T, W>::at(row, 4 * c + 2 * h));
        const f32x4 hi = *(const f32x4 *)(tile + Tile<T, W>::at(row, 4 * c + 2 * h + 1));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// Fragment across rows: eight rows, 16 c + 8 (j / 4) + 4 h + j % 4, of column col0 + lane % 32.  bf16: ds_read_b64_tr_b16, in
// which 16 lanes read 4 rows of 16 columns (lane i the columns 4 (i % 4) .. of row i / 4) and get one column of 4 rows each.
template <typename T, int W>
__device__ __forceinline__ typename Frag<T>::type load_t(const char *tile, int c, int col0)
{
    const int l = threadIdx.x & 63, h = l >> 5;
    if constexpr (sizeof(T) == 2) {
        const int i = l & 15, col = col0 + (l >> 4 & 1) * 16 + (i & 3) * 4;
        s16x4 v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int row = 16 * c + 8 * k + 4 * h + (i >> 2);
            const char *p = tile + Tile<T, W>::at(row, col >> 3) + (col & 7) * 2;
            v[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KT_LDS s16x4 *)p);
        }
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        const int col = col0 + (l & 31);
        f32x8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = 16 * c + 8 * (j >> 2) + 4 * h + (j & 3);
            v[j] = *(const float *)(tile + Tile<T, W>::at(row, col >> 2) + (col & 3) * 4);
        }
        return v;
    }
}

}  // namespace

#endif
