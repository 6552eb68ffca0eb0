// Activation checkpoints in 8 bits: save and restore.
//
// Both are one pass over the data, bound by memory: save reads s and writes 1.03 bytes an element, restore the
// other way round.  A lane holds 16 bytes of the wide side (8 bf16 or 4 f32), so that the wide accesses of a wavefront are
// 1 KiB in one piece; the 4 or 8 lanes of a group find its largest magnitude in the vector pipe.
// Rows need not start at multiples of 16 bytes: the wide side is accessed at any element address.
// The wide side is read and written past the caches (non-temporal) where its rows start at multiples of 16 bytes: 16 384 x 8 192
// bf16 saved in 61 us (6.6 TB/s; plain loads 72 to 84), restored in 60 (plain stores 71).  Elsewhere neighbouring lanes share a
// line, which would be fetched twice.
#include "kt_ops_device.h"

namespace {

constexpr int BLOCK = 256;
constexpr int PER = 4;            // chunks per lane, all loaded before the first is used

// n / d for n < 2^31 by one multiplication: m = ceil(2^(31 + l) / d), l = ceil(log2 d).
struct Div {
    uint32_t m, shift, d;
    static Div by(uint32_t d)
    {
        uint32_t l = 0;
        while ((1ull << l) < d) ++l;
        return Div{(uint32_t)(((1ull << (31 + l)) + d - 1) / d), 31 + l, d};
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

// Chunks are numbered over rows of `per_row`, the padding of the last group among them.
template <typename T, bool NT>
__global__ __launch_bounds__(BLOCK) void kt_act8_save_kernel(const T *x, int64_t ldx, int8_t *q, uint8_t *e, int cols,
                                                             uint32_t total, Div per_row)
{
    constexpr int V = VE<T>;
    const uint32_t n0 = blockIdx.x * (BLOCK * PER) + threadIdx.x;
    u32x4 r[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const uint32_t n = n0 + u * BLOCK, row = per_row(n), c = (n - row * per_row.d) * V;
        r[u] = n < total ? ld_chunk<T, NT>(x + (int64_t)row * ldx, (int)c, cols) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const uint32_t n = n0 + u * BLOCK;
        float f[V];
        widen<T>(r[u], f);
        const Step s = group_step(group_max<V>(f));
        uint32_t w[V / 4];
        to_bytes<V>(f, s, w);
        if (n < total) {
            if constexpr (V == 8) *(u32x2 *)(q + (uint64_t)n * V) = u32x2{w[0], w[1]};
            else *(uint32_t *)(q + (uint64_t)n * V) = w[0];
            if (n % (KT_ACT8_GROUP / V) == 0) e[n / (KT_ACT8_GROUP / V)] = (uint8_t)s.e;
        }
    }
}

template <typename T, bool NT>
__global__ __launch_bounds__(BLOCK) void kt_act8_restore_kernel(const int8_t *q, const uint8_t *e, T *y, int64_t ldy, int cols,
                                                                uint32_t total, Div per_row)
{
    constexpr int V = VE<T>;
    const uint32_t n0 = blockIdx.x * (BLOCK * PER) + threadIdx.x;
    uint32_t w[PER][V / 4], eb[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const uint32_t n = min(n0 + u * BLOCK, total - 1);
        if constexpr (V == 8) {
            const u32x2 v = *(const u32x2 *)(q + (uint64_t)n * V);
            w[u][0] = v[0];
            w[u][1] = v[1];
        } else {
            w[u][0] = *(const uint32_t *)(q + (uint64_t)n * V);
        }
        eb[u] = e[n / (KT_ACT8_GROUP / V)];
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const uint32_t n = n0 + u * BLOCK;
        if (n >= total) break;
        const uint32_t row = per_row(n), c = (n - row * per_row.d) * V;
        float f[V];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) from_bytes(w[u][j], step_of(eb[u]), f + 4 * j);
        st_chunk<T, NT>(y + (int64_t)row * ldy, (int)c, cols, narrow<T>(f));
    }
}

// Calls f(first row, rows) for pieces whose chunks can be numbered in 31 bits with room for a workgroup beyond the last.
template <typename F> int in_pieces(int64_t rows, int64_t per_row, F f)
{
    const int64_t most = ((1ll << 31) - BLOCK * PER) / per_row;
    for (int64_t r = 0; r < rows; r += most) {
        const int e = f(r, rows - r < most ? rows - r : most);
        if (e) return e;
    }
    return 0;
}

template <typename T>
int save(int64_t rows, int64_t cols, const T *x, int64_t ldx, int8_t *q, uint8_t *e, hipStream_t s)
{
    const int64_t G = kt_act8_groups(cols), per_row = G * (KT_ACT8_GROUP / VE<T>);
    return in_pieces(rows, per_row, [&](int64_t r, int64_t n) {
        const uint32_t total = (uint32_t)(n * per_row);
        const unsigned grid = (total + BLOCK * PER - 1) / (BLOCK * PER);
        auto kernel = rows_of_16(x, ldx) ? kt_act8_save_kernel<T, true> : kt_act8_save_kernel<T, false>;
        kernel<<<grid, BLOCK, 0, s>>>(x + r * ldx, ldx, q + r * G * KT_ACT8_GROUP, e + r * G, (int)cols, total, Div::by((uint32_t)per_row));
        return (int)hipGetLastError();
    });
}

template <typename T>
int restore(int64_t rows, int64_t cols, const int8_t *q, const uint8_t *e, T *y, int64_t ldy, hipStream_t s)
{
    const int64_t G = kt_act8_groups(cols), per_row = G * (KT_ACT8_GROUP / VE<T>);
    return in_pieces(rows, per_row, [&](int64_t r, int64_t n) {
        const uint32_t total = (uint32_t)(n * per_row);
        const unsigned grid = (total + BLOCK * PER - 1) / (BLOCK * PER);
        auto kernel = rows_of_16(y, ldy) ? kt_act8_restore_kernel<T, true> : kt_act8_restore_kernel<T, false>;
        kernel<<<grid, BLOCK, 0, s>>>(q + r * G * KT_ACT8_GROUP, e + r * G, y + r * ldy, ldy, (int)cols, total, Div::by((uint32_t)per_row));
        return (int)hipGetLastError();
    });
}

}  // namespace

int kt_launch_act8_save(kt_dtype dt, int64_t rows, int64_t cols, const void *x, int64_t ldx, int8_t *q, uint8_t *e,
                        void *stream)
{
    if (dt == KT_F32) return save(rows, cols, (const float *)x, ldx, q, e, (hipStream_t)stream);
    return save(rows, cols, (const bf16 *)x, ldx, q, e, (hipStream_t)stream);
}

int kt_launch_act8_restore(kt_dtype dt, int64_t rows, int64_t cols, const int8_t *q, const uint8_t *e, void *y,
                           int64_t ldy, void *stream)
{
    if (dt == KT_F32) return restore(rows, cols, q, e, (float *)y, ldy, (hipStream_t)stream);
    return restore(rows, cols, q, e, (bf16 *)y, ldy, (hipStream_t)stream);
}
