// Embedding lookup y[t] = scale * w[id_t], and its gradient dw[v] = scale * sum over the tokens t with id_t = v of dy[t].
//
// The lookup moves rows and memory bounds it: a wavefront takes a row's next 4 KiB, all of its loads on their way at once.  16384 rows of 2048 bf16, 92 MB:
// 17 us with the table's rows in the last-level cache, 21 in a sequence of other passes (4.3 TB/s); a single row 4.2, the launch.
//
// The gradient adds rows in the order of (id, t), whatever the chip does first: the tokens are sorted by their id (stable, digits
// from the lowest up), the sorted list is cut into pieces of equal length, and a wavefront adds a piece's rows, a row of the table
// for every id in it.  So a token that fills half of the batch costs no more than others.  A run of equal ids that crosses pieces
// leaves partial sums, which a last kernel adds in their order.  Rows without a token are zeros, written (all rows are) beside the
// sort, which takes few workgroups and much waiting.
// Memory bounds it too.  16384 tokens, 50304 x 2048 bf16, 273 MB: 67 to 75 us, 3.7 to 4.1 TB/s (two passes of the sort 44, in which 206 MB of zeros are
// written; sums 22, joins 6); 65536 tokens, half of them one: 115 to 129 (sort 41, sums 74, joins 10).
#include "kt_ops_device.h"

namespace {

constexpr int64_t MOST_BLOCKS = 1 << 20;        // of a launch; what is more is taken in turns

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }

template <typename I> __device__ __forceinline__ int key_of(I id, int vocab)
{
    return id >= 0 && id < (I)vocab ? (int)id : vocab;      // sorted behind all others
}

// E neighbouring elements of a row from column c on, as binary32; what lies past `cols` is 0 and is not read.
template <typename T, int E> __device__ __forceinline__ void load_e(const T *row, int64_t c, int64_t cols, u32x4 *r)
{
#pragma unroll
    for (int k = 0; k < E / VE<T>; ++k) {
        const int64_t at = c + k * VE<T>;
        r[k] = at < cols ? ld_chunk(row + at, 0, (int)min((int64_t)VE<T>, cols - at)) : u32x4{0, 0, 0, 0};
    }
}
template <typename T, int E> __device__ __forceinline__ void widen_e(const u32x4 *r, float *f)
{
#pragma unroll
    for (int k = 0; k < E / VE<T>; ++k) widen<T>(r[k], f + k * VE<T>);
}
template <typename T, int E> __device__ __forceinline__ void store_e(T *row, int64_t c, int64_t cols, const float *f)
{
#pragma unroll
    for (int k = 0; k < E / VE<T>; ++k) {
        const int64_t at = c + k * VE<T>;
        if (at < cols) st_chunk(row + at, 0, (int)min((int64_t)VE<T>, cols - at), narrow<T>(f + k * VE<T>));
    }
}
// Elements that a lane takes of a row: 16 bytes of the narrower type.
template <typename T, typename W> constexpr int EACH = VE<T> > VE<W> ? VE<T> : VE<W>;

// ---- lookup ----------------------------------------------------------------------

constexpr int SPANS = 4;        // of 64 lanes that a wavefront takes of a row

template <typename T, typename W, typename I>
__global__ __launch_bounds__(256) void kt_embedding_fwd_kernel(const I *ids, const W *w, int64_t ldw, T *y, int64_t ldy, float scale,
                                                               int64_t items, int parts, int vocab, int width)
{
    constexpr int E = EACH<T, W>, R = E / VE<W>;
    for (int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; n < items; n += (int64_t)gridDim.x * 4) {
        const int64_t t = n / parts;
        const int key = key_of(ids[t], vocab), c0 = (int)(n % parts) * (SPANS * 64 * E) + (threadIdx.x & 63) * E;
        const W *row = w + key * ldw;
        u32x4 r[SPANS][R];
#pragma unroll
        for (int s = 0; s < SPANS; ++s) {
#pragma unroll
            for (int k = 0; k < R; ++k) r[s][k] = u32x4{0, 0, 0, 0};
            if (key < vocab) load_e<W, E>(row, c0 + s * 64 * E, width, r[s]);
        }
#pragma unroll
        for (int s = 0; s < SPANS; ++s) {
            float f[E];
            widen_e<W, E>(r[s], f);
#pragma unroll
            for (int j = 0; j < E; ++j) f[j] = key < vocab ? f[j] * scale : 0.0f;
            store_e<T, E>(y + t * ldy, c0 + s * 64 * E, width, f);
        }
    }
}

template <typename T, typename W, typename I>
int fwd(int64_t tokens, int vocab, int width, const I *ids, const W *w, int64_t ldw, float scale, T *y, int64_t ldy, hipStream_t s)
{
    constexpr int each = SPANS * 64 * EACH<T, W>;
    const int parts = (width + each - 1) / each;
    const int64_t items = tokens * parts, blocks = (items + 3) / 4;
    kt_embedding_fwd_kernel<T, W, I><<<(unsigned)(blocks < MOST_BLOCKS ? blocks : MOST_BLOCKS), 256, 0, s>>>(ids, w, ldw, y, ldy, scale, items, parts, vocab, width);
    return (int)hipGetLastError();
}

// ---- zeros beside the sort ---------------------------------------------------------

// The part-th 4 KiB of a row of `bytes` bytes, by a wavefront.
__device__ __forceinline__ void fill_part(char *row, int64_t part, int64_t bytes, int lane)
{
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int64_t at = part * 4096 + s * 1024 + lane * 16;
        if (at + 16 <= bytes) st16(row + at, u32x4{0, 0, 0, 0});
        else
            for (int64_t b = at; b < bytes; b += 2) *(uint16_t *)(row + b) = 0;
    }
}
// A share of a matrix to fill with zeros: items [from, to) of 4 KiB of a row each.
struct Fill {
    char *p;
    int64_t ld, row, parts, from, to;           // bytes; items to a row
};
// `block` of `blocks` workgroups of `lanes`.
__device__ __forceinline__ void fill(const Fill &f, int block, int blocks, int lanes)
{
    const int lane = threadIdx.x & 63, waves = lanes / 64;
    for (int64_t n = f.from + (int64_t)block * waves + threadIdx.x / 64; n < f.to; n += (int64_t)blocks * waves) {
        fill_part(f.p + n / f.parts * f.ld, n % f.parts, f.row, lane);
    }
}

// ---- sorting the tokens by their id ------------------------------------------------

// Lanes of this wavefront whose digit is this lane's, `active` lanes only.
__device__ __forceinline__ uint64_t same_digit(int digit, int bits, uint64_t active)
{
    uint64_t m = active;
    for (int b = 0; b < bits; ++b) {
        const uint64_t on = __ballot(digit >> b & 1);
        m &= digit >> b & 1 ? on : ~on;
    }
    return m;
}
__device__ __forceinline__ int lanes_below(uint64_t m)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}
// This lane's place among those with its digit; `next` (LDS, of this wavefront alone) holds the first free place of each digit and moves on.
__device__ __forceinline__ int place_of(int digit, int bits, bool active, volatile int *next)
{
    const uint64_t act = __ballot(active), m = same_digit(digit, bits, act);
    const int below = lanes_below(m);
    int first = 0;
    if (active) first = next[digit];
    __builtin_amdgcn_wave_barrier();            // all lanes have read before the first one writes
    if (active && below == 0) next[digit] = first + __popcll(m);
    __builtin_amdgcn_wave_barrier();
    return first + below;
}
// Exclusive sums of `n` numbers in LDS in place, by all lanes of the workgroup (at most n of them work); `carry`: LDS, 16 numbers.
__device__ __forceinline__ void exclusive_sums(int *x, int n, int *carry)
{
    const int lanes = blockDim.x, tid = threadIdx.x;
    int before = 0;
    for (int at = 0; at < n; at += lanes) {
        const int v = at + tid < n ? x[at + tid] : 0;
        int s = v;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(s, d);
            if ((tid & 63) >= d) s += o;
        }
        if ((tid & 63) == 63) carry[tid / 64] = s;
        __syncthreads();
        int below = before, all = before;
        for (int w = 0; w < lanes / 64; ++w) {
            if (w < tid / 64) below += carry[w];
            all += carry[w];
        }
        if (at + tid < n) x[at + tid] = below + s - v;
        before = all;
        __syncthreads();
    }
}

// Up to FEW tokens: one workgroup sorts them in LDS, the others fill.
constexpr int FEW = 4096, FEW_LANES = 1024, FEW_WAVES = FEW_LANES / 64, FEW_EACH = FEW / FEW_LANES, FEW_BITS = 8;

template <typename I>
__global__ __launch_bounds__(FEW_LANES) void kt_embedding_sort_few_kernel(const I *ids, int *keys, int *order, int tokens, int vocab, int bits,
                                                                          Fill zeros)
{
    if (blockIdx.x > 0) {
        fill(zeros, blockIdx.x - 1, gridDim.x - 1, FEW_LANES);
        return;
    }
    constexpr int BINS = 1 << FEW_BITS;
    __shared__ int key[FEW], pos[FEW], next[FEW_WAVES][BINS], total[BINS], carry[16];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
    // a wavefront's elements are neighbours, 64 of them a round
    const int rounds = (tokens + FEW_LANES - 1) / FEW_LANES, first = wave * rounds * 64;
    int k[FEW_EACH], p[FEW_EACH];
#pragma unroll
    for (int r = 0; r < FEW_EACH; ++r) {
        const int at = first + r * 64 + lane;
        p[r] = at;
        k[r] = r < rounds && at < tokens ? key_of(ids[at], vocab) : 0;
    }
    for (int shift = 0; shift < bits; shift += FEW_BITS) {
        for (int i = tid; i < FEW_WAVES * BINS; i += FEW_LANES) (&next[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < FEW_EACH; ++r)
            if (r < rounds && first + r * 64 + lane < tokens) atomicAdd(&next[wave][k[r] >> shift & (BINS - 1)], 1);
        __syncthreads();
        if (tid < BINS) {
            int s = 0;
            for (int w = 0; w < FEW_WAVES; ++w) s += next[w][tid];
            total[tid] = s;
        }
        __syncthreads();
        exclusive_sums(total, BINS, carry);
        if (tid < BINS) {
            int s = total[tid];
            for (int w = 0; w < FEW_WAVES; ++w) {
                const int n = next[w][tid];
                next[w][tid] = s;
                s += n;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < FEW_EACH; ++r) {
            if (r >= rounds) break;
            const bool on = first + r * 64 + lane < tokens;
            const int to = place_of(k[r] >> shift & (BINS - 1), FEW_BITS, on, next[wave]);
            if (on) {
                key[to] = k[r];
                pos[to] = p[r];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < FEW_EACH; ++r) {
            const int at = first + r * 64 + lane;
            if (r < rounds && at < tokens) {
                k[r] = key[at];
                p[r] = pos[at];
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < FEW_EACH; ++r) {
        const int at = first + r * 64 + lane;
        if (r < rounds && at < tokens) {
            keys[at] = k[r];
            order[at] = p[r];
        }
    }
}

// More tokens: a workgroup has a stretch of them; a pass over one digit is two kernels, the first of which counts.
constexpr int LANES = 1024, WAVES = LANES / 64, STRETCH = 2 * LANES, MOST_BITS = 9, MOST_BINS = 1 << MOST_BITS;

// What a pass reads: the ids as they are, or what the last pass left.
template <typename I, bool FIRST> struct Source {
    const I *ids;
    const int *keys, *order;
    __device__ __forceinline__ int key(int64_t n, int vocab) const
    {
        if constexpr (FIRST) return key_of(ids[n], vocab);
        else return keys[n];
    }
    __device__ __forceinline__ int pos(int64_t n) const
    {
        if constexpr (FIRST) return (int)n;
        else return order[n];
    }
};

// counts[block][digit]
template <typename I, bool FIRST>
__global__ __launch_bounds__(LANES) void kt_embedding_count_kernel(Source<I, FIRST> from, int *counts, int tokens, int vocab, int stretch,
                                                                   int stretches, int shift, int bits, Fill zeros)
{
    if ((int)blockIdx.x >= stretches) {
        fill(zeros, blockIdx.x - stretches, gridDim.x - stretches, LANES);
        return;
    }
    __shared__ int count[MOST_BINS];
    const int bins = 1 << bits;
    for (int i = threadIdx.x; i < bins; i += LANES) count[i] = 0;
    __syncthreads();
    const int64_t n0 = (int64_t)blockIdx.x * stretch, n1 = min((int64_t)tokens, n0 + stretch);
    for (int64_t n = n0 + threadIdx.x; n < n1; n += LANES) atomicAdd(&count[from.key(n, vocab) >> shift & (bins - 1)], 1);
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += LANES) counts[blockIdx.x * bins + i] = count[i];
}

template <typename I, bool FIRST>
__global__ __launch_bounds__(LANES) void kt_embedding_place_kernel(Source<I, FIRST> from, const int *counts, int *keys, int *order, int tokens,
                                                                   int vocab, int stretch, int stretches, int shift, int bits, Fill zeros)
{
    if ((int)blockIdx.x >= stretches) {
        fill(zeros, blockIdx.x - stretches, gridDim.x - stretches, LANES);
        return;
    }
    __shared__ int next[WAVES][MOST_BINS], total[MOST_BINS], before[MOST_BINS], carry[16];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63, bins = 1 << bits;
    for (int i = tid; i < bins; i += LANES) total[i] = before[i] = 0;
    for (int i = lane; i < bins; i += 64) next[wave][i] = 0;
    __syncthreads();
    // a wavefront's elements are neighbours
    const int64_t each = stretch / WAVES, n0 = min((int64_t)tokens, (int64_t)blockIdx.x * stretch + wave * each), n1 = min((int64_t)tokens, n0 + each);
    for (int64_t n = n0 + lane; n < n1; n += 64) atomicAdd(&next[wave][from.key(n, vocab) >> shift & (bins - 1)], 1);
    // of each digit: all of them, and those in the stretches before this one
    int all = 0, mine = 0;
#pragma unroll 4
    for (int b = tid >> bits; b < stretches; b += LANES >> bits) {
        const int n = counts[b * bins + (tid & (bins - 1))];
        all += n;
        mine += b < (int)blockIdx.x ? n : 0;
    }
    atomicAdd(&total[tid & (bins - 1)], all);
    atomicAdd(&before[tid & (bins - 1)], mine);
    __syncthreads();
    exclusive_sums(total, bins, carry);
    if (tid < bins) {
        int s = total[tid] + before[tid];
        for (int w = 0; w < WAVES; ++w) {
            const int n = next[w][tid];
            next[w][tid] = s;
            s += n;
        }
    }
    __syncthreads();
    for (int64_t n = n0; n < n1; n += 64) {
        const bool on = n + lane < n1;
        const int key = on ? from.key(n + lane, vocab) : 0;
        const int to = place_of(key >> shift & (bins - 1), bits, on, next[wave]);
        if (on) {
            keys[to] = key;
            order[to] = from.pos(n + lane);
        }
    }
}

// ---- sums ------------------------------------------------------------------------

// Writes a row's sum.
template <typename W, int E, bool ADD> __device__ __forceinline__ void put(W *row, int64_t c, int width, float scale, const float *sum)
{
    float f[E];
#pragma unroll
    for (int j = 0; j < E; ++j) f[j] = sum[j] * scale;
    if constexpr (ADD) {
        u32x4 old[E / VE<W>];
        float o[E];
        load_e<W, E>(row, c, width, old);
        widen_e<W, E>(old, o);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");         // a neighbour may write what this lane reads (Columns): no load sinks below the first store
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] += o[j];
    }
    store_e<W, E>(row, c, width, f);
}

// E columns for each lane of a wavefront, from column c0 on.  A lane whose columns end past the row takes the row's last E instead, some of them as its neighbour
// does: both write the same numbers, with one instruction.  (Not the first lane: its neighbour is another wavefront.)  Lanes past the row
// read what the first one does.
template <int E> struct Columns {
    bool whole;                 // E columns from `from` on are there in every lane
    int c, from;
    __device__ __forceinline__ Columns(int c0, int lane, int width) : whole(c0 + E <= width), c(c0 + lane * E)
    {
        if (whole && c < width) c = min(c, width - E);
        from = c < width ? c : c0;
    }
};

constexpr int AHEAD = 8;        // rows on their way at once

// A wavefront adds the rows of a piece of the sorted list, 64 * E columns of them, eight rows' loads on their way while eight are added.  parts[piece][0]: the sum of what a run that began
// before the piece has in it; [1]: of a run that begins in it and goes on behind it.
template <typename T, typename W, bool ADD>
__global__ __launch_bounds__(256) void kt_embedding_sum_kernel(const int *keys, const int *order, const T *dy, int64_t lddy, W *dw, int64_t lddw,
                                                               float *parts, int ldp, float scale, int tokens, int vocab, int width, int piece,
                                                               int pieces, int spans)
{
    constexpr int E = EACH<T, W>, R = E / VE<T>;
    const int lane = threadIdx.x & 63;
    const int64_t n = (int64_t)blockIdx.x * 4 + wave_of();
    if (n >= (int64_t)pieces * spans) return;
    const int p = (int)(n / spans), c0 = (int)(n % spans) * (64 * E);
    const Columns<E> at(c0, lane, width);
    const int c = at.c;
    const int i0 = p * piece, i1 = min(tokens, i0 + piece);
    const int before = i0 ? keys[i0 - 1] : -1, behind = i1 < tokens ? keys[i1] : -1;
    float sum[E];
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] = 0.0f;
    int now = -1;                               // the key whose rows `sum` holds
    bool begun = false;                         // before this piece
    auto end = [&](bool goes_on) {
        if (begun || goes_on) {
            float *to = parts + ((int64_t)p * 2 + (begun ? 0 : 1)) * ldp;
            if (c < width) {
#pragma unroll
                for (int j = 0; j < E; j += 4) *(u32x4_any *)(to + c + j) = u32x4{as_u(sum[j]), as_u(sum[j + 1]), as_u(sum[j + 2]), as_u(sum[j + 3])};
            }
        } else {
            put<W, E, ADD>(dw + now * lddw, c, width, scale, sum);
        }
    };
    for (int i = i0; i < i1; i += 64) {
        const int mine = min(i + lane, i1 - 1), key = keys[mine], pos = order[mine], count = min(64, i1 - i);
        auto load = [&](u32x4 (&r)[AHEAD][R], int a) __attribute__((always_inline)) {
            if (at.whole && a + AHEAD <= count && __builtin_amdgcn_readlane(key, a + AHEAD - 1) < vocab) {
                // without a branch, so that the loads leave together
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const T *row = dy + (int64_t)__builtin_amdgcn_readlane(pos, a + u) * lddy + at.from;
#pragma unroll
                    for (int k = 0; k < R; ++k) r[u][k] = ld16<true>(row + k * VE<T>);
                }
            } else {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int l = min(a + u, count - 1);
                    const T *row = dy + (int64_t)__builtin_amdgcn_readlane(pos, l) * lddy;
                    if (a + u < count && __builtin_amdgcn_readlane(key, l) < vocab) load_e<T, E>(row, c, width, r[u]);
                }
            }
        };
        auto use = [&](const u32x4 (&r)[AHEAD][R], int a) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (a + u >= count) break;
                const int k = __builtin_amdgcn_readlane(key, a + u);
                if (k != now) {
                    if (now >= 0) end(false);
                    now = k < vocab ? k : -1;
                    begun = k == before;
#pragma unroll
                    for (int j = 0; j < E; ++j) sum[j] = 0.0f;
                }
                if (now >= 0) {
                    float f[E];
                    widen_e<T, E>(r[u], f);
#pragma unroll
                    for (int j = 0; j < E; ++j) sum[j] += f[j];
                }
            }
        };
        u32x4 r0[AHEAD][R], r1[AHEAD][R];       // one is on its way while the other is added
        load(r0, 0);
        for (int a = 0; a < count; a += 2 * AHEAD) {
            if (a + AHEAD < count) load(r1, a + AHEAD);
            use(r0, a);
            if (a + 2 * AHEAD < count) load(r0, a + 2 * AHEAD);
            if (a + AHEAD < count) use(r1, a + AHEAD);
        }
    }
    if (now >= 0) end(now == behind);
}

// A run that begins in piece p and goes on behind it: the partial sums in their order.  Each wavefront has a piece, and adds what its run left if that
// is up to SHORT partial sums; all of them add a longer one together, each a stretch of it.
constexpr int JOIN = 512, JOIN_WAVES = JOIN / 64, SHORT = 16;

template <typename W, bool ADD>
__global__ __launch_bounds__(JOIN) void kt_embedding_join_kernel(const int *keys, const float *parts, int ldp, W *dw, int64_t lddw, float scale,
                                                                 int vocab, int width, int piece, int pieces)
{
    __shared__ int run[JOIN_WAVES], key_of_run[JOIN_WAVES];                     // pieces behind the one that it begins in
    __shared__ __align__(16) float sums[JOIN_WAVES][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, p0 = blockIdx.x * JOIN_WAVES, p = p0 + wave;
    int n = 0, key = -1;
    if (p < pieces - 1) {                               // not the last piece: there are tokens behind it
        const int i0 = p * piece, i1 = i0 + piece;
        key = keys[i1 - 1];
        if (key < vocab && keys[i1] == key && !(i0 && keys[i0 - 1] == key)) {
            int q = p + 1;                              // to the first piece that does not begin with the key
            for (;;) {
                const int at = q + lane;
                const uint64_t other = __ballot(at >= pieces || keys[(int64_t)at * piece] != key);
                if (other) {
                    q += __builtin_ctzll(other);
                    break;
                }
                q += 64;
            }
            n = q - p - 1;
        }
    }
    if (lane == 0) {
        run[wave] = n;
        key_of_run[wave] = key;
    }
    __syncthreads();
    auto add = [&](float (&s)[4], u32x4 r) {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += as_f(r[j]);
    };
    // the first partial sums of pieces a to b - 1, LOADS of them on their way at once
    auto add_all = [&](float (&s)[4], int a, int b, int c) {
        constexpr int LOADS = 16;
        for (; a < b; a += LOADS) {
            u32x4 r[LOADS];
#pragma unroll
            for (int u = 0; u < LOADS; ++u) r[u] = *(const u32x4 *)(parts + (int64_t)min(a + u, b - 1) * 2 * ldp + c);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < LOADS; ++u)
                if (a + u < b) add(s, r[u]);
        }
    };
    auto put4 = [&](int k, int c, const float (&s)[4]) {
        typedef W W4 __attribute__((ext_vector_type(4)));
        typedef W4 W4_any __attribute__((aligned(sizeof(W))));
        W *row = dw + (int64_t)k * lddw + c;
        if (c + 4 <= width) {
            W4 v;
            if (ADD) v = *(const W4_any *)row;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (W)(s[j] * scale + (ADD ? (float)v[j] : 0.0f));
            *(W4_any *)row = v;
        } else {
            for (int j = 0; j < width - c; ++j) row[j] = (W)(s[j] * scale + (ADD ? (float)row[j] : 0.0f));
        }
    };
    for (int c0 = blockIdx.y * 256; c0 < width; c0 += gridDim.y * 256) {
        const int c = c0 + lane * 4;
        if (n > 0 && n <= SHORT && c < width) {
            float s[4] = {0, 0, 0, 0};
            add(s, *(const u32x4 *)(parts + ((int64_t)p * 2 + 1) * ldp + c));
            add_all(s, p + 1, p + 1 + n, c);
            put4(key, c, s);
        }
        for (int r = 0; r < JOIN_WAVES; ++r) {
            const int m = run[r];
            if (m <= SHORT) continue;
            const int each = (m + JOIN_WAVES - 1) / JOIN_WAVES, a = p0 + r + 1 + wave * each, b = min(p0 + r + 1 + m, a + each);
            float s[4] = {0, 0, 0, 0};
            if (c < width) {
                if (wave == 0) add(s, *(const u32x4 *)(parts + ((int64_t)(p0 + r) * 2 + 1) * ldp + c));
                add_all(s, a, b, c);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[wave][lane * 4 + j] = s[j];
            __syncthreads();
            if (wave == 0 && c < width) {
                for (int w = 1; w < JOIN_WAVES; ++w)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[j] += sums[w][lane * 4 + j];
                put4(key_of_run[r], c, s);
            }
            __syncthreads();
        }
    }
}

// ---- a handful of tokens -------------------------------------------------------------
//
// Up to HANDFUL tokens need no order: every wavefront has all ids in four registers.  That of a token's first occurrence adds its rows, those of the
// other occurrences have nothing to do; the wavefronts behind them write zeros into the rows whose number is not among the ids.  One launch
// instead of three: 197 tokens of 1000 x 768 f32 15.0 -> 6.3 us.
constexpr int HANDFUL = 256;

template <typename T, typename W, typename I, bool ADD>
__global__ __launch_bounds__(256) void kt_embedding_handful_kernel(const I *ids, const T *dy, int64_t lddy, W *dw, int64_t lddw, float scale, int tokens,
                                                                   int vocab, int width, int spans)
{
    constexpr int E = EACH<T, W>, R = E / VE<T>, WORDS = HANDFUL / 64;
    const int lane = threadIdx.x & 63;
    int key[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) key[w] = w * 64 + lane < tokens ? key_of(ids[w * 64 + lane], vocab) : vocab;
    const int64_t waves = (int64_t)gridDim.x * 4, sums = (int64_t)tokens * spans;
    int64_t n = (int64_t)blockIdx.x * 4 + wave_of();
    if (n < sums) {
        const int t = (int)(n / spans), c0 = (int)(n % spans) * (64 * E);
        int mine = vocab;
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
            if (w == t / 64) mine = __builtin_amdgcn_readlane(key[w], t % 64);
        uint64_t same[WORDS];
        bool first = mine < vocab;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            same[w] = __ballot(key[w] == mine);
            if (w < t / 64 ? same[w] != 0 : w == t / 64 && (same[w] & ((1ull << t % 64) - 1))) first = false;
        }
        if (first) {
            const Columns<E> at(c0, lane, width);
            float sum[E];
#pragma unroll
            for (int j = 0; j < E; ++j) sum[j] = 0.0f;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                uint64_t left = same[w];
                while (left) {
                    u32x4 r[AHEAD][R];
                    const int there = min(AHEAD, __popcll(left));
                    int l = 0;
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        if (left) l = __builtin_ctzll(left);            // else the last one again
                        left &= left - 1;
                        const T *row = dy + (int64_t)(w * 64 + l) * lddy;
                        if (at.whole) {
#pragma unroll
                            for (int k = 0; k < R; ++k) r[u][k] = ld16<true>(row + at.from + k * VE<T>);
                        } else {
                            load_e<T, E>(row, at.c, width, r[u]);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        if (u >= there) break;
                        float f[E];
                        widen_e<T, E>(r[u], f);
#pragma unroll
                        for (int j = 0; j < E; ++j) sum[j] += f[j];
                    }
                }
            }
            put<W, E, ADD>(dw + (int64_t)mine * lddw, at.c, width, scale, sum);
        }
        return;
    }
    if (ADD) return;
    const int64_t row_bytes = width * (int64_t)sizeof(W), parts = (row_bytes + 4095) / 4096;
    for (n -= sums; n < vocab * parts; n += waves - sums) {
        const int64_t v = n / parts;
        bool named = false;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) named |= key[w] == (int)v;
        if (__ballot(named) == 0) fill_part((char *)(dw + v * lddw), n % parts, row_bytes, lane);
    }
}

// ---- how the gradient is cut ---------------------------------------------------------

struct Cut {
    int piece, pieces, ldp;                     // of the sorted list; floats to a partial sum
    int bits, passes, stretch, stretches;       // of the sort
    int64_t lists, counts, bytes;               // in the workspace: one list; the counts; all of it
};
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int bits_of(int64_t n)
{
    int b = 0;
    while (n >> b) ++b;
    return b;
}
// 8 rows to a piece, and at most 2^20 / width pieces within 512 to 2 048.  More make more partial sums, fewer too few wavefronts: 65536 tokens of 50304 x 2048
// bf16, half of them one, 115 us in 512, 120 in 1 024, 134 in 2 048; 60000 of 131072 x 768 bf16 into f32 126, 116 and 119.
Cut cut(int64_t tokens, int64_t vocab, int64_t width)
{
    Cut c{};
    int64_t most = (1 << 20) / width;
    most = most < 512 ? 512 : most > 2048 ? 2048 : most;
    c.piece = (int)((tokens + most - 1) / most);
    if (c.piece < 8) c.piece = 8;
    c.pieces = (int)((tokens + c.piece - 1) / c.piece);
    c.ldp = (int)up(width, 8);
    const int all = bits_of(vocab);             // `vocab` itself stands for no token
    c.passes = (all + MOST_BITS - 1) / MOST_BITS;
    c.bits = (all + c.passes - 1) / c.passes;
    c.stretch = (int)up((tokens + 511) / 512, LANES);
    if (c.stretch < STRETCH) c.stretch = STRETCH;
    c.stretches = (int)((tokens + c.stretch - 1) / c.stretch);
    c.lists = up(tokens * 4, 256);
    c.counts = tokens <= FEW ? 0 : up((int64_t)c.stretches * 4 << c.bits, 256);
    c.bytes = tokens <= HANDFUL ? 0 : (tokens <= FEW ? 2 : 4) * c.lists + c.counts + (c.pieces > 1 ? (int64_t)c.pieces * 2 * c.ldp * 4 : 0);
    return c;
}

template <typename I, bool FIRST>
int pass(const Cut &c, const Source<I, FIRST> &from, int *counts, int *keys, int *order, int tokens, int vocab, int shift, const Fill &f1,
         const Fill &f2, hipStream_t s)
{
    auto blocks = [&](const Fill &f) {
        const int64_t n = (f.to - f.from + 63) / 64;
        return (unsigned)(c.stretches + (n < 512 ? n : 512));
    };
    kt_embedding_count_kernel<I, FIRST><<<blocks(f1), LANES, 0, s>>>(from, counts, tokens, vocab, c.stretch, c.stretches, shift, c.bits, f1);
    kt_embedding_place_kernel<I, FIRST><<<blocks(f2), LANES, 0, s>>>(from, counts, keys, order, tokens, vocab, c.stretch, c.stretches, shift, c.bits, f2);
    return (int)hipGetLastError();
}

template <typename T, typename W, bool ADD>
int sums(const Cut &c, const int *keys, const int *order, const T *dy, int64_t lddy, W *dw, int64_t lddw, float *parts, float scale, int tokens,
         int vocab, int width, hipStream_t s)
{
    constexpr int span = 64 * EACH<T, W>;
    const int spans = (width + span - 1) / span;
    const int64_t waves = (int64_t)c.pieces * spans;
    kt_embedding_sum_kernel<T, W, ADD><<<(unsigned)((waves + 3) / 4), 256, 0, s>>>(keys, order, dy, lddy, dw, lddw, parts, c.ldp, scale, tokens, vocab, width, c.piece, c.pieces, spans);
    if (c.pieces > 1) {
        const int across = (width + 255) / 256;
        kt_embedding_join_kernel<W, ADD><<<dim3((c.pieces - 1 + JOIN_WAVES - 1) / JOIN_WAVES, across < 64 ? across : 64), JOIN, 0, s>>>(keys, parts, c.ldp, dw, lddw, scale, vocab, width, c.piece, c.pieces);
    }
    return (int)hipGetLastError();
}

template <typename T, typename W, typename I>
int bwd(int64_t tokens, int vocab, int width, const I *ids, const T *dy, int64_t lddy, float scale, W *dw, int64_t lddw, bool add, char *ws,
        hipStream_t s)
{
    if (tokens <= HANDFUL) {
        const int span = 64 * EACH<T, W>, spans = (width + span - 1) / span;
        const int64_t zeros = add ? 0 : vocab * ((width * (int64_t)sizeof(W) + 4095) / 4096);
        const int64_t waves = tokens * spans + (zeros < 65536 ? zeros : 65536);
        if (waves == 0) return 0;
        // (a wavefront of zeros at least, whatever the last workgroup leaves of them)
        const unsigned blocks = (unsigned)((waves + 3) / 4);
        if (add) kt_embedding_handful_kernel<T, W, I, true><<<blocks, 256, 0, s>>>(ids, dy, lddy, dw, lddw, scale, (int)tokens, vocab, width, spans);
        else kt_embedding_handful_kernel<T, W, I, false><<<blocks, 256, 0, s>>>(ids, dy, lddy, dw, lddw, scale, (int)tokens, vocab, width, spans);
        return (int)hipGetLastError();
    }
    const Cut c = cut(tokens, vocab, width);
    // zeros: a share of them beside every kernel of the sort
    Fill all{(char *)dw, lddw * (int64_t)sizeof(W), width * (int64_t)sizeof(W), 1, 0, 0};
    int64_t rows = vocab;
    if (lddw == width) {
        all.row *= vocab;
        rows = 1;
    }
    all.parts = (all.row + 4095) / 4096;
    const int64_t items = add ? 0 : rows * all.parts;
    auto share = [&](int k, int of) {
        Fill f = all;
        f.from = items * k / of;
        f.to = items * (k + 1) / of;
        return f;
    };
    int *list[4];
    for (int i = 0; i < 4; ++i) list[i] = (int *)(ws + i * c.lists);
    int *keys = list[0], *order = list[1];
    if (tokens <= FEW) {
        const Fill f = share(0, 1);
        const int64_t n = (f.to - f.from + 63) / 64;
        kt_embedding_sort_few_kernel<I><<<(unsigned)(1 + (n < 512 ? n : 512)), FEW_LANES, 0, s>>>(ids, keys, order, (int)tokens, vocab, bits_of(vocab), f);
        if (const int e = (int)hipGetLastError()) return e;
    } else {
        int *counts = (int *)(ws + 4 * c.lists);
        const int of = 2 * c.passes;
        // the last pass ends in the first two lists
        int to = c.passes % 2 ? 0 : 2;
        int e = pass(c, Source<I, true>{ids, nullptr, nullptr}, counts, list[to], list[to + 1], (int)tokens, vocab, 0, share(0, of), share(1, of), s);
        for (int k = 1; k < c.passes && !e; ++k, to = 2 - to)
            e = pass(c, Source<I, false>{nullptr, list[to], list[to + 1]}, counts, list[2 - to], list[3 - to], (int)tokens, vocab, k * c.bits, share(2 * k, of),
                     share(2 * k + 1, of), s);
        if (e) return e;
    }
    float *parts = (float *)(ws + (tokens <= FEW ? 2 : 4) * c.lists + c.counts);
    if (add) return sums<T, W, true>(c, keys, order, dy, lddy, dw, lddw, parts, scale, (int)tokens, vocab, width, s);
    return sums<T, W, false>(c, keys, order, dy, lddy, dw, lddw, parts, scale, (int)tokens, vocab, width, s);
}

// f(T, W, I): values of the types.
template <typename F> int by_types(kt_dtype dt, kt_dtype wdt, kt_index it, F f)
{
    auto index = [&](auto t, auto w) { return it == KT_I32 ? f(t, w, int32_t()) : f(t, w, int64_t()); };
    auto table = [&](auto t) { return wdt == KT_F32 ? index(t, float()) : index(t, bf16()); };
    return dt == KT_F32 ? table(float()) : table(bf16());
}

}  // namespace

int64_t kt_embedding_bwd_ws(int64_t tokens, int64_t vocab, int64_t width) { return cut(tokens, vocab, width).bytes; }

int kt_launch_embedding_fwd(kt_dtype dt, kt_dtype wdt, kt_index it, int64_t tokens, int vocab, int width, const void *ids, const void *w,
                            int64_t ldw, float scale, void *y, int64_t ldy, void *stream)
{
    return by_types(dt, wdt, it, [&](auto t, auto u, auto i) {
        return fwd(tokens, vocab, width, (const decltype(i) *)ids, (const decltype(u) *)w, ldw, scale, (decltype(t) *)y, ldy, (hipStream_t)stream);
    });
}

int kt_launch_embedding_bwd(kt_dtype dt, kt_dtype wdt, kt_index it, int64_t tokens, int vocab, int width, const void *ids, const void *dy,
                            int64_t lddy, float scale, void *dw, int64_t lddw, bool add, void *ws, void *stream)
{
    return by_types(dt, wdt, it, [&](auto t, auto u, auto i) {
        return bwd(tokens, vocab, width, (const decltype(i) *)ids, (const decltype(t) *)dy, lddy, scale, (decltype(u) *)dw, lddw, add, (char *)ws, (hipStream_t)stream);
    });
}
