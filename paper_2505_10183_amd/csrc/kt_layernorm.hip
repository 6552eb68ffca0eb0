// Layer norm, forward and backward, with the reduction of the gradients of weight and bias.
//
// Both are one pass over the rows, bound by memory: a row is held in registers by LANES lanes (16 bytes a chunk, NV
// chunks a lane), so that mean, squared deviations and output need one read; gamma and beta stay in registers over the
// rows that a workgroup takes, and the next row is on its way while one is worked on.  A wavefront takes a
// row of up to 2 048 (bf16) or 1 024 (f32) columns by itself: its sums cross lanes in the vector pipe, without LDS or
// barriers.  Wider rows take 4 or 16 wavefronts.
//
// The backward pass keeps dy * xh and dy of its columns in registers over all rows of the workgroup; a workgroup writes one
// partial sum per column, and a second kernel adds these in a fixed order.
//
// Measured (kernel trace; data that was used just before is partly in the last-level cache): forward with checkpoint, 16384 x 2048 bf16 30 us
// (170 MB, 5.6 TB/s; 39 amid a block's training step); backward 25216 x 768 f32 39 us and 5 for the sums (6.0 TB/s), 9001 x 1001 bf16 through
// a checkpoint 15 and 4 (3.0 TB/s: rows that start at odd addresses), 16384 x 2048 bf16 through a checkpoint 41 with the sums, 27 at 6.33
// TB/s.  197 x 768 f32 is one launch, 4 us.
//
// Wide rows in the backward pass hold more than registers do: with 1 024 lanes 14 to 231 registers are spilled for f32, 28 to 56 for bf16 (8192 x
// 8192 f32 148 us, 5.4 TB/s; 4096 x 16384 f32 319 us, 2.5, bf16 135, 3.0).
#include "kt_ops_device.h"

namespace {

constexpr int ROW_WAVES = 4;      // wavefronts of a workgroup that takes one row per wavefront
constexpr int MAX_NV = 4;

template <int LANES> constexpr int WAVES = LANES / 64;                    // that share a row
template <int LANES> constexpr int ROWS = LANES == 64 ? ROW_WAVES : 1;    // rows that a workgroup takes at a time
template <int LANES> constexpr int BLOCK = LANES * ROWS<LANES>;

template <typename T, typename P> __device__ __forceinline__ void load_param(const P *p, int c, int cols, float *f)
{
    constexpr int V = VE<T>;
    if constexpr (V == VE<P>) {
        widen<P>(ld_chunk(p, c, cols), f);
    } else if constexpr (V > VE<P>) {                      // 8 columns of f32
        widen<P>(ld_chunk(p, c, cols), f);
        widen<P>(ld_chunk(p, c + 4, cols), f + 4);
    } else {                                               // 4 columns of bf16
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = c + j < cols ? (float)p[c + j] : 0.0f;
    }
}

template <typename T, typename P, int LANES, int NV, bool SAVE>
__global__ __launch_bounds__(BLOCK<LANES>) void kt_layernorm_fwd_kernel(const T *x, int64_t ldx, const P *gamma,
                                                                        const P *beta, T *y, int64_t ldy, float *mean,
                                                                        float *rstd, int8_t *y8, uint8_t *e8, int64_t rows,
                                                                        int cols, float eps)
{
    constexpr int V = VE<T>;
    __shared__ float red[2 * WAVES<LANES>];
    const int lane = threadIdx.x % LANES, groups = (cols + KT_ACT8_GROUP - 1) / KT_ACT8_GROUP;
    const int64_t step = (int64_t)gridDim.x * ROWS<LANES>;
    int64_t row = (int64_t)blockIdx.x * ROWS<LANES> + threadIdx.x / LANES;
    const float n_cols = (float)cols;          // divided by: 1 / cols would add a rounding to every row's mean and rstd
    float g[NV][V], b[NV][V];
    u32x4 next[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) next[i] = row < rows ? ld_chunk(x + row * ldx, (i * LANES + lane) * V, cols) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_param<T, P>(gamma, (i * LANES + lane) * V, cols, g[i]);
        if (beta) {
            load_param<T, P>(beta, (i * LANES + lane) * V, cols, b[i]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) b[i][j] = 0.0f;
        }
    }
    // with several wavefronts to a row all of a workgroup's leave the loop together: one row at a time
    for (; row < rows; row += step) {
        float f[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) widen<T>(next[i], f[i]);
        if (row + step < rows) {
#pragma unroll
            for (int i = 0; i < NV; ++i) next[i] = ld_chunk(x + (row + step) * ldx, (i * LANES + lane) * V, cols);
        }
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] += f[i][j];
        row_sum<WAVES<LANES>>(s, red, 0);
        const float mu = s[0] / n_cols;
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int n = cols - (i * LANES + lane) * V;
            if (n >= V) {
#pragma unroll
                for (int j = 0; j < V; ++j) { f[i][j] -= mu; s[0] = __fmaf_rn(f[i][j], f[i][j], s[0]); }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) { f[i][j] = j < n ? f[i][j] - mu : 0.0f; s[0] = __fmaf_rn(f[i][j], f[i][j], s[0]); }
            }
        }
        row_sum<WAVES<LANES>>(s, red, 1);
        const float rs = 1.0f / __fsqrt_rn(s[0] / n_cols + eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LANES + lane) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) f[i][j] = __fmaf_rn(f[i][j] * rs, g[i][j], b[i][j]);
            const u32x4 out = narrow<T>(f[i]);
            st_chunk<T, true>(y + row * ldy, c, cols, out);
            if constexpr (SAVE) {           // of the values that y keeps; columns past the last are 0: g = b = 0
                widen<T>(out, f[i]);
                if (c >= cols) {
#pragma unroll
                    for (int j = 0; j < V; ++j) f[i][j] = 0.0f;      // not a NaN row's 0 * NaN
                } else if (c + V > cols) {
#pragma unroll
                    for (int j = 0; j < V; ++j) f[i][j] = c + j < cols ? f[i][j] : 0.0f;
                }
                const Step st = group_step(group_max<V>(f[i]));
                uint32_t w[V / 4];
                to_bytes<V>(f[i], st, w);
                if (c < groups * KT_ACT8_GROUP) {
                    int8_t *q = y8 + row * ((int64_t)groups * KT_ACT8_GROUP) + c;
                    if constexpr (V == 8) *(u32x2 *)q = u32x2{w[0], w[1]};
                    else *(uint32_t *)q = w[0];
                    if (c % KT_ACT8_GROUP == 0) e8[row * groups + c / KT_ACT8_GROUP] = (uint8_t)st.e;
                }
            }
        }
        if (lane == 0 && mean) { mean[row] = mu; rstd[row] = rs; }
    }
}

// One row's dy and x as they lie in memory.
template <typename T, int NV, bool X8> struct RowIn {
    static constexpr int V = VE<T>;
    u32x4 dy[NV];
    u32x4 x[X8 ? 1 : NV];
    uint32_t w[X8 ? NV : 1][V / 4];
    uint32_t e[X8 ? NV : 1];
    float mu, rs;
};

template <typename T, typename P, int LANES, int NV, bool X8, bool NT>
__global__ __launch_bounds__(BLOCK<LANES>) void kt_layernorm_bwd_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                                        const int8_t *x8, const uint8_t *e8, const P *gamma,
                                                                        const float *mean, const float *rstd, T *dx,
                                                                        int64_t lddx, float *parts, int64_t rows, int cols,
                                                                        int pcols)
{
    constexpr int V = VE<T>;
    constexpr int ACROSS = LANES == 64 ? ROW_WAVES * 64 * V * 2 : 1;
    __shared__ float red[4 * WAVES<LANES>];
    __shared__ float across[ACROSS];
    const int lane = threadIdx.x % LANES, groups = (cols + KT_ACT8_GROUP - 1) / KT_ACT8_GROUP;
    const int64_t step = (int64_t)gridDim.x * ROWS<LANES>;
    int64_t row = (int64_t)blockIdx.x * ROWS<LANES> + threadIdx.x / LANES;
    const float n_cols = (float)cols;          // divided by, as in the forward pass
    float g[NV][V], dg[NV][V], db[NV][V];
    auto load = [&](int64_t r, RowIn<T, NV, X8> &in) {
        in.mu = mean[r];
        in.rs = rstd[r];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LANES + lane) * V;
            in.dy[i] = ld_chunk<T, NT>(dy + r * lddy, c, cols);
            if constexpr (X8) {
                in.e[i] = 0;
#pragma unroll
                for (int j = 0; j < V / 4; ++j) in.w[i][j] = 0;
                if (c < groups * KT_ACT8_GROUP) {
                    const int8_t *q = x8 + r * ((int64_t)groups * KT_ACT8_GROUP) + c;
                    if constexpr (V == 8) {
                        const u32x2 v = *(const u32x2 *)q;
                        in.w[i][0] = v[0];
                        in.w[i][1] = v[1];
                    } else {
                        in.w[i][0] = *(const uint32_t *)q;
                    }
                    in.e[i] = e8[r * groups + c / KT_ACT8_GROUP];
                }
            } else {
                in.x[i] = ld_chunk<T, NT>(x + r * ldx, c, cols);
            }
        }
    };
    RowIn<T, NV, X8> next;
    if (row < rows) load(row, next);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_param<T, P>(gamma, (i * LANES + lane) * V, cols, g[i]);
#pragma unroll
        for (int j = 0; j < V; ++j) dg[i][j] = db[i][j] = 0.0f;
    }
    int turn = 0;
    for (; row < rows; row += step, turn ^= 1) {
        RowIn<T, NV, X8> in = next;
        if (row + step < rows) load(row + step, next);
        float xh[NV][V], t[NV][V], s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            widen<T>(in.dy[i], t[i]);
            if constexpr (X8) {
#pragma unroll
                for (int j = 0; j < V / 4; ++j) from_bytes(in.w[i][j], step_of(in.e[i]), xh[i] + 4 * j);
            } else {
                widen<T>(in.x[i], xh[i]);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                xh[i][j] = (xh[i][j] - in.mu) * in.rs;
                db[i][j] += t[i][j];
                dg[i][j] = __fmaf_rn(t[i][j], xh[i][j], dg[i][j]);
                t[i][j] *= g[i][j];              // columns past the last: dy = 0
                s[0] += t[i][j];
                s[1] = __fmaf_rn(t[i][j], xh[i][j], s[1]);
            }
        }
        row_sum<WAVES<LANES>>(s, red, turn);
        const float m1 = s[0] / n_cols, m2 = s[1] / n_cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < V; ++j) t[i][j] = (t[i][j] - __fmaf_rn(xh[i][j], m2, m1)) * in.rs;
            st_chunk<T, true>(dx + row * lddx, (i * LANES + lane) * V, cols, narrow<T>(t[i]));
        }
    }
    float *pg = parts + (int64_t)blockIdx.x * 2 * pcols, *pb = pg + pcols;
    if constexpr (LANES == 64) {
        // the four wavefronts' sums, chunk by chunk, in the order of the wavefronts
        const int wave = threadIdx.x / 64;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                across[((wave * 2 + 0) * V + j) * 64 + lane] = dg[i][j];
                across[((wave * 2 + 1) * V + j) * 64 + lane] = db[i][j];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 2 * V / ROW_WAVES; ++k) {
                const int n = k * ROW_WAVES + wave;                 // dg of V columns, then db
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < ROW_WAVES; ++w) s += across[(w * 2 * V + n) * 64 + lane];
                const int c = (i * 64 + lane) * V + n % V;
                if (c < cols) (n < V ? pg : pb)[c] = s;
            }
            __syncthreads();
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = (i * LANES + lane) * V + j;
                if (c < cols) { pg[c] = dg[i][j]; pb[c] = db[i][j]; }
            }
    }
}

// Sums of the workgroups' partial results: 64 columns to a workgroup, its 16 wavefronts take every 16th part and are added
// in their order.  Rows of columns are read whole: 256 bytes a wavefront and part.
constexpr int SUM_WAVES = 16;
template <typename P>
__global__ __launch_bounds__(64 * SUM_WAVES) void kt_layernorm_sum_kernel(const float *parts, int n, int cols, int pcols, P *dgamma,
                                                                          P *dbeta)
{
    __shared__ float across[SUM_WAVES][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int c = blockIdx.x * 64 + lane;                           // of [dgamma | dbeta]
    float s = 0.0f;
    if (c < 2 * pcols) {
        const float *p = parts + c;
#pragma unroll 8
        for (int i = wave; i < n; i += SUM_WAVES) s += p[(int64_t)i * 2 * pcols];
    }
    across[wave][lane] = s;
    __syncthreads();
    if (wave) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < SUM_WAVES; ++w) s += across[w][lane];
    if (c < cols) dgamma[c] = (P)s;
    else if (c >= pcols && c < pcols + cols && dbeta) dbeta[c - pcols] = (P)s;
}

// f with N lanes and `nv` chunks a lane, at least NV of them: the kernels for the most columns that N lanes can have, and no more.
template <typename T, int N, int NV, typename F> int with_chunks(int nv, F f)
{
    constexpr int MOST = (KT_LAYERNORM_MAX_COLS / VE<T> + N - 1) / N;
    if constexpr (NV < MAX_NV && NV < MOST)
        if (nv > NV) return with_chunks<T, N, NV + 1>(nv, f);
    return f(std::integral_constant<int, N>(), std::integral_constant<int, NV>());
}
// Lanes and chunks for a row: the fewest lanes that hold it in MAX_NV chunks each.  With four times the lanes of the step below a row has
// two chunks or more.
template <typename T, typename F> int with_shape(int cols, F f)
{
    const int chunks = (cols + VE<T> - 1) / VE<T>;
    if (chunks <= 64 * MAX_NV) return with_chunks<T, 64, 1>((chunks + 63) / 64, f);
    if (chunks <= 256 * MAX_NV) return with_chunks<T, 256, 2>((chunks + 255) / 256, f);
    return with_chunks<T, 1024, 2>((chunks + 1023) / 1024, f);
}
static_assert(1024 * MAX_NV * VE<float> >= KT_LAYERNORM_MAX_COLS, "f32 rows need more lanes");

template <typename T, typename P>
int fwd(int64_t rows, int cols, const T *x, int64_t ldx, const P *gamma, const P *beta, float eps, T *y, int64_t ldy,
        float *mean, float *rstd, int8_t *y8, uint8_t *e8, hipStream_t s)
{
    return with_shape<T>(cols, [&](auto L, auto N) {
        constexpr int LANES = decltype(L)::value, NV = decltype(N)::value;
        const int64_t need = (rows + ROWS<LANES> - 1) / ROWS<LANES>;
        const unsigned grid = (unsigned)(need < 2048 ? need : 2048);
        if (y8)
            kt_layernorm_fwd_kernel<T, P, LANES, NV, true><<<grid, BLOCK<LANES>, 0, s>>>(x, ldx, gamma, beta, y, ldy, mean, rstd, y8, e8, rows, cols, eps);
        else
            kt_layernorm_fwd_kernel<T, P, LANES, NV, false><<<grid, BLOCK<LANES>, 0, s>>>(x, ldx, gamma, beta, y, ldy, mean, rstd, nullptr, nullptr, rows, cols, eps);
        return (int)hipGetLastError();
    });
}

int padded(int cols) { return (cols + 63) / 64 * 64; }

template <typename T, typename P>
int bwd(int64_t rows, int cols, const T *dy, int64_t lddy, const T *x, int64_t ldx, const int8_t *x8, const uint8_t *e8,
        const P *gamma, const float *mean, const float *rstd, T *dx, int64_t lddx, P *dgamma, P *dbeta, float *ws,
        hipStream_t s)
{
    const int parts = (int)kt_layernorm_bwd_parts(rows, cols), pcols = padded(cols);
    if (parts) {
        const int e = with_shape<T>(cols, [&](auto L, auto N) {
            constexpr int LANES = decltype(L)::value, NV = decltype(N)::value;
            const bool nt = rows_of_16(dy, lddy) && (x8 || rows_of_16(x, ldx));
            auto kernel = x8 ? (nt ? kt_layernorm_bwd_kernel<T, P, LANES, NV, true, true> : kt_layernorm_bwd_kernel<T, P, LANES, NV, true, false>)
                             : (nt ? kt_layernorm_bwd_kernel<T, P, LANES, NV, false, true> : kt_layernorm_bwd_kernel<T, P, LANES, NV, false, false>);
            kernel<<<parts, BLOCK<LANES>, 0, s>>>(dy, lddy, x, ldx, x8, e8, gamma, mean, rstd, dx, lddx, ws, rows, cols, pcols);
            return (int)hipGetLastError();
        });
        if (e) return e;
    }
    kt_layernorm_sum_kernel<P><<<(2 * pcols + 63) / 64, 64 * SUM_WAVES, 0, s>>>(ws, parts, cols, pcols, dgamma, dbeta);
    return (int)hipGetLastError();
}

}  // namespace

// Workgroups of the backward pass, each with one partial sum per column: two to a CU, fewer where they would have under 16 rows each, which
// is 4 to a wavefront where a wavefront takes a row.  Where several take one, a workgroup has its 16 rows one after another, and few rows
// leave most of the chip idle: 1 000 rows of 8 192 are 63 workgroups, 38 us in bf16 for 8 at 6.33 TB/s.
int64_t kt_layernorm_bwd_parts(int64_t rows, int64_t)
{
    const int64_t need = (rows + 15) / 16;
    return need < 512 ? need : 512;
}

extern "C" int64_t kt_layernorm_bwd_workspace(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1 || cols > KT_LAYERNORM_MAX_COLS) return 0;
    return kt_layernorm_bwd_parts(rows, cols) * 2 * padded((int)cols) * (int64_t)sizeof(float);
}

int kt_launch_layernorm_fwd(kt_dtype dt, kt_dtype pdt, int64_t rows, int cols, const void *x, int64_t ldx,
                            const void *gamma, const void *beta, float eps, void *y, int64_t ldy, float *mean,
                            float *rstd, int8_t *y8, uint8_t *e8, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    auto go = [&](auto *t, auto *p) {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(p)> P;
        return fwd<T, P>(rows, cols, (const T *)x, ldx, (const P *)gamma, (const P *)beta, eps, (T *)y, ldy, mean, rstd, y8, e8, s);
    };
    if (dt == KT_F32) return pdt == KT_F32 ? go((float *)0, (float *)0) : go((float *)0, (bf16 *)0);
    return pdt == KT_F32 ? go((bf16 *)0, (float *)0) : go((bf16 *)0, (bf16 *)0);
}

int kt_launch_layernorm_bwd(kt_dtype dt, kt_dtype pdt, int64_t rows, int cols, const void *dy, int64_t lddy,
                            const void *x, int64_t ldx, const int8_t *x8, const uint8_t *e8, const void *gamma,
                            const float *mean, const float *rstd, void *dx, int64_t lddx, void *dgamma, void *dbeta,
                            float *ws, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    auto go = [&](auto *t, auto *p) {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(p)> P;
        return bwd<T, P>(rows, cols, (const T *)dy, lddy, (const T *)x, ldx, x8, e8, (const P *)gamma, mean, rstd, (T *)dx, lddx,
                         (P *)dgamma, (P *)dbeta, ws, s);
    };
    if (dt == KT_F32) return pdt == KT_F32 ? go((float *)0, (float *)0) : go((float *)0, (bf16 *)0);
    return pdt == KT_F32 ? go((bf16 *)0, (float *)0) : go((bf16 *)0, (bf16 *)0);
}
