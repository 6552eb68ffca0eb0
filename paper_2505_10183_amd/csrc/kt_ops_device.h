// Device-side helpers of the operators: 16-byte chunks of a row as binary32 values, sums over a wavefront, the
// 8-bit groups of a checkpoint.  Internal to a translation unit (anonymous namespace).
#ifndef KT_OPS_DEVICE_H
#define KT_OPS_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kt_ops_internal.h"

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// 16 bytes at any element address: one global_load/store_dwordx4 each (kernels run in unaligned access mode).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

namespace {

typedef __bf16 bf16;

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }
// Two values rounded to bf16, nearest-even, in one word (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// A chunk: the 16 bytes of a row that one lane holds.
template <typename T> constexpr int VE = 16 / (int)sizeof(T);

template <typename T> __device__ __forceinline__ void widen(u32x4 r, float *f);
template <> __device__ __forceinline__ void widen<float>(u32x4 r, float *f)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = as_f(r[j]);
}
template <> __device__ __forceinline__ void widen<bf16>(u32x4 r, float *f)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) { f[2 * j] = as_f(r[j] << 16); f[2 * j + 1] = as_f(r[j] & 0xffff0000u); }
}
template <typename T> __device__ __forceinline__ u32x4 narrow(const float *f);
template <> __device__ __forceinline__ u32x4 narrow<float>(const float *f)
{
    return u32x4{as_u(f[0]), as_u(f[1]), as_u(f[2]), as_u(f[3])};
}
template <> __device__ __forceinline__ u32x4 narrow<bf16>(const float *f)
{
    return u32x4{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])};
}

// NT: non-temporal, for data that streams through once.
template <bool NT = false> __device__ __forceinline__ u32x4 ld16(const void *p)
{
    if constexpr (NT) return __builtin_nontemporal_load((const u32x4_any *)p);
    else return *(const u32x4_any *)p;
}
template <bool NT = false> __device__ __forceinline__ void st16(void *p, u32x4 v)
{
    if constexpr (NT) __builtin_nontemporal_store(v, (u32x4_any *)p);
    else *(u32x4_any *)p = v;
}
// Whether rows start at multiples of 16 bytes.
template <typename T> bool rows_of_16(const T *p, int64_t ld)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (int64_t)sizeof(T) % 16 == 0;
}

// The chunk of a row that starts at column c; columns at and past `cols` read as 0 and are not stored.
template <typename T, bool NT = false> __device__ __forceinline__ u32x4 ld_chunk(const T *row, int c, int cols)
{
    if (c + VE<T> <= cols) return ld16<NT>(row + c);
    u32x4 r{0, 0, 0, 0};
    if (c < cols) {
#pragma unroll
        for (int j = 0; j < VE<T>; ++j) {
            if (c + j < cols) {
                if (sizeof(T) == 4) r[j & 3] = ((const uint32_t *)row)[c + j];
                else r[j / 2] |= (uint32_t)((const uint16_t *)row)[c + j] << (16 * (j & 1));
            }
        }
    }
    return r;
}
template <typename T, bool NT = false> __device__ __forceinline__ void st_chunk(T *row, int c, int cols, u32x4 v)
{
    if (c + VE<T> <= cols) { st16<NT>(row + c, v); return; }
#pragma unroll
    for (int j = 0; j < VE<T>; ++j) {
        if (c + j < cols) {
            if (sizeof(T) == 4) ((uint32_t *)row)[c + j] = v[j & 3];
            else ((uint16_t *)row)[c + j] = (uint16_t)(v[j / 2] >> (16 * (j & 1)));
        }
    }
}

// ---- over a wavefront ------------------------------------------------------------

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// Sum over the 64 lanes, the same in all of them: neighbours, quads, rows of 16 in the vector pipe, then
// halves by lane swaps; no LDS.
__device__ __forceinline__ float wave_sum(float x)
{
    x += as_f(dpp<DPP_XOR1>(as_u(x)));
    x += as_f(dpp<DPP_XOR2>(as_u(x)));
    x += as_f(dpp<DPP_HALF_MIRROR>(as_u(x)));
    x += as_f(dpp<DPP_MIRROR>(as_u(x)));
    auto a = __builtin_amdgcn_permlane16_swap(as_u(x), as_u(x), false, false);
    x = as_f(a[0]) + as_f(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
    return as_f(b[0]) + as_f(b[1]);
}

// Sums of N values over the WAVES wavefronts of a workgroup that share a row; `at` is the half of `red` (2 x N x WAVES
// floats) that this reduction uses: taking turns, one barrier is enough.
template <int WAVES, int N> __device__ __forceinline__ void row_sum(float (&x)[N], float *red, int at)
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
    if constexpr (WAVES > 1) {
        float *r = red + at * N * WAVES;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i * WAVES + threadIdx.x / 64] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = r[i * WAVES];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += r[i * WAVES + w];
            x[i] = s;
        }
    }
}

// ---- groups of a checkpoint ------------------------------------------------------

// The largest magnitude (as bits: NaN above infinity above all numbers) over the lanes that share a group of 32
// columns: 4 lanes of 8 columns or 8 lanes of 4.
template <int V> __device__ __forceinline__ uint32_t group_max(const float *f)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) m = max(m, as_u(f[j]) & 0x7fffffffu);
    m = max(m, dpp<DPP_XOR1>(m));
    m = max(m, dpp<DPP_XOR2>(m));
    if (V == 4) m = max(m, dpp<DPP_HALF_MIRROR>(m));
    return m;
}

// The scale byte of a group and the factor 2^(127 - e) that makes steps of its members.
struct Step {
    uint32_t e;
    float up;
};
__device__ __forceinline__ Step group_step(uint32_t largest)
{
    const int power = (int)(largest >> 23);
    Step s;
    s.e = power == 255 ? 255u : (uint32_t)max(power - 6, 1);
    s.up = power == 255 ? 0.0f : as_f((254u - s.e) << 23);
    return s;
}
// V members as bytes.  x * up is exact (a power of two), so the one rounding is that of the addition: 1.5 * 2^23 has
// unit 1 in its last place, which leaves rint(x * up), ties to even, in the low byte.  A group that is not finite has up = 0:
// 0 * inf = NaN, which the clamp turns into an end of the range; those bytes are cleared.
template <int V> __device__ __forceinline__ void to_bytes(const float *f, const Step &s, uint32_t *w)
{
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = as_u(__builtin_amdgcn_fmed3f(f[j + i] * s.up, -127.0f, 127.0f) + 12582912.0f);
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
        w[j / 4] = s.e == 255 ? 0u : lo | hi << 16;
    }
}
// The values that 4 bytes with scale byte e stand for: q * 2^(e - 127); e = 255 gives 0 * inf = NaN, e = 0 gives 0.
__device__ __forceinline__ float step_of(uint32_t e) { return as_f(e << 23); }
__device__ __forceinline__ void from_bytes(uint32_t w, float step, float *f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i)) * step;
}

}  // namespace

#endif
