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

#include <type_traits>
#include <utility>

#include "kt_ops_device.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define KT_LDS __attribute__((address_space(3)))

namespace {

// f(A), f(A + 1), ... f(B - 1), the numbers known to the compiler.
template <int A, typename F, int... I> __device__ __forceinline__ void span_of(F f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, A + I>()), ...);
}
template <int A, int B, typename F> __device__ __forceinline__ void span(F f)
{
    if constexpr (A < B) span_of<A>(f, std::make_integer_sequence<int, B - A>());
}

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

// The wavefront's number, known to be the same in all of its lanes: what follows from it are scalars and scalar branches.
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }

// 16 bytes, or one byte, at `at` of a buffer of `bytes` bytes; zeros where it ends before.
__device__ __forceinline__ u32x4 buffer16([[maybe_unused]] const void *p, [[maybe_unused]] int bytes, [[maybe_unused]] int at)
{
#ifdef __HIP_DEVICE_COMPILE__           // the host pass knows neither the type nor the builtins
    return __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000), at, 0, 0);
#else
    return u32x4{0, 0, 0, 0};
#endif
}
__device__ __forceinline__ uint32_t buffer1([[maybe_unused]] const void *p, [[maybe_unused]] int bytes, [[maybe_unused]] int at)
{
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_raw_buffer_load_b8(__builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000), at, 0, 0);
#else
    return 0;
#endif
}

// Tiles of R rows of D elements on their way from memory to LDS, brought by BLOCK lanes; rows at and past `end` are zeros and are not read.
// DMA: the loads write LDS themselves, 16 bytes a lane, without a register: lane l of an instruction writes the l-th 16 bytes of
// a KiB, so the exchange of chunks (Tile) is made on the side of the addresses.  The buffer's size ends at the last row, which
// makes zeros of what lies past it; columns past dim are sent there too.  It needs rows at multiples of 16 bytes and offsets
// within a tile of 31 bits; other tensors pass through registers.
template <typename T, int D, int R, int BLOCK, bool DMA> struct Feed {
    static constexpr int V = VE<T>, N = R * D / V / BLOCK;
    static_assert(N >= 1, "a tile has a chunk for every lane");
    const T *p;
    int64_t stride;
    int end, dim;
    u32x4 r[DMA ? 1 : N];
    int at[DMA ? N : 1];

    __device__ __forceinline__ Feed(const T *p_, int64_t stride_, int end_, int dim_) : p(p_), stride(stride_), end(end_), dim(dim_)
    {
        if constexpr (DMA) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int n = threadIdx.x + u * BLOCK, row = n / (D / V), c = (n % (D / V) ^ Tile<T, D>::swizzle(row)) * V;
                at[u] = c < dim ? row * (int)stride * (int)sizeof(T) + c * (int)sizeof(T) : INT32_MIN;
            }
        }
    }
    // In assembly: of the builtin the compiler only knows that it writes LDS some time, and waits for it before the next read of
    // any tile.  The instruction has no output register and reads its operands when it is issued; arrived() waits for it.  s_nop: m0
    // and a descriptor that the vector unit has just written need up to 5 cycles before a memory instruction reads them.  m0 cannot
    // be named as overwritten (it is reserved); nothing else in these kernels uses it.
    __device__ __forceinline__ void bring(const T *from, int bytes, char *tile) const
    {
        const uint64_t base = (uint64_t)from;
        const u32x4 rs{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, (uint32_t)bytes, 0x00020000u};
        const uint32_t to = (uint32_t)(uintptr_t)(KT_LDS char *)tile + wave_id() * 1024;
#pragma unroll
        for (int u = 0; u < N; ++u)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                         :: "s"(to + u * BLOCK * 16), "v"(at[u]), "s"(rs) : "memory");
    }
    // Starts bringing the rows from row0 on into `tile`; they are there after finish() and a barrier.
    __device__ __forceinline__ void start(char *tile, int row0)
    {
        if constexpr (DMA) {
            const int rows = min(R, end - row0);
            const int bytes = rows > 0 ? ((rows - 1) * (int)stride + dim) * (int)sizeof(T) : 0;
            bring(p + row0 * stride, bytes, tile);
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int n = threadIdx.x + u * BLOCK, row = row0 + n / (D / V);
                r[u] = row < end ? ld_chunk(p + row * stride, n % (D / V) * V, dim) : u32x4{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void finish(char *tile) const
    {
        if constexpr (!DMA) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int n = threadIdx.x + u * BLOCK;
                *(u32x4 *)(tile + Tile<T, D>::at(n / (D / V), n % (D / V))) = r[u];
            }
        }
    }
};
// Before the barrier behind which a tile is read: what this wavefront brings has arrived.
// LATER: loads started after it that may still be on their way.
template <int LATER = 0> __device__ __forceinline__ void arrived()
{
    static_assert(LATER < 16, "the low four bits of vmcnt");
    asm volatile("" ::: "memory");          // the later loads stay before it: LATER counts them
    __builtin_amdgcn_s_waitcnt(0x0f70 | LATER);
    asm volatile("" ::: "memory");
}

}  // namespace

#endif
