// The weight gradient of a linear layer from the 8-bit checkpoint of its input: dw[o][i] = sum_t dy[t][o] x8[t][i].
//
// Both operands run over t along their rows, so both are read across rows from LDS.  A workgroup makes a tile of BM x BN of dw: per
// step, K rows of dy and of x8 go from memory into registers one or two steps before they are needed, x8 is turned into
// dy's type on its way into LDS (exact in bf16: 7 bits and a power of two), and the two halves of LDS take turns, one barrier
// a step.  Rows of dy at multiples of 16 bytes are brought into LDS by the loads themselves (Feed).  Both the conversion and the
// reads of the next fragments stand beside the products (sched_barrier): the matrix cores take 32 cycles for one, in which a
// wavefront issues 8 other instructions.  Where dw has too few tiles for the chip, t is cut into pieces whose sums a second kernel
// adds in their order.
//
// Bound by the matrix cores and the clock they leave: 16384 x 2048 x 8192 bf16 468 to 499 us with the card, 1.10 to 1.17 PFLOP/s (a library
// product of the same sizes from bf16 in memory 554 us); they are busy 58 % of the cycles, LDS 37 % (7 % of them bank conflicts).  Few tiles
// are bound by one workgroup's steps one after another: 4099 x 1001 x 4004 has 256 tiles of 128, 65 us; 197 x 768 x 768 f32 144 of 64, 10 us.
// (Passes among others, by events; a kernel trace shows 508 and 74 us.)
#include "kt_mfma.h"

namespace {

// Tile and wavefronts: WM x WN of them, each FM x FN products of 32 x 32; rows of bf16 a step (half as many of f32) with dy brought
// by DMA, and through registers.
template <int WM_, int WN_, int FM_, int FN_, int KD, int KR> struct Shape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32, BLOCK = WM * WN * 64;
    template <typename T, bool DMA> static constexpr int K = (DMA ? KD : KR) * 2 / (int)sizeof(T);
};
typedef Shape<2, 4, 4, 2, 64, 32> Big;      // 256 x 256, 8 wavefronts, 128 or 64 KiB of LDS
typedef Shape<2, 2, 2, 2, 64, 64> Mid;      // 128 x 128, 4,  64 KiB
typedef Shape<2, 2, 1, 1, 64, 64> Small;    //  64 x  64, 4,  32 KiB

// Tile of a workgroup: those of one XCD (every eighth workgroup) are neighbours, dy's columns first, so that its L2 keeps a
// strip of x8 and all of dy's current rows.
__device__ __forceinline__ int xcd_order(int b, int n)
{
    const int q = n / 8, r = n % 8, x = b % 8;
    return x * q + min(x, r) + b / 8;
}

template <typename T, typename S, typename G, bool PIECES, bool DMA>
__global__ __launch_bounds__(S::BLOCK) void kt_weight_grad_kernel(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e,
                                                                  G *dw, int64_t lddw, int64_t tokens, int out, int in, int mt,
                                                                  int64_t piece)
{
    constexpr int K = S::template K<T, DMA>, V = VE<T>;
    constexpr int AC = DMA ? 0 : K * S::BM / V / S::BLOCK;  // 16-byte chunks of dy that pass through a lane
    constexpr int BC = K * S::BN / 16 / S::BLOCK > 0 ? K * S::BN / 16 / S::BLOCK : 1;        // 16 bytes of x8 each
    constexpr bool BPART = K * S::BN / 16 < S::BLOCK;       // the first lanes only
    constexpr int BU = 16 / V;                              // 16-byte chunks in LDS that 16 bytes of x8 make
    typedef Tile<T, S::BM> TA;
    typedef Tile<T, S::BN> TB;
    typedef typename Frag<T>::type F;
    constexpr int HALF = TA::bytes(K) + TB::bytes(K);
    extern __shared__ __align__(16) char lds[];             // two halves

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid & 63;
    const int tile = xcd_order(blockIdx.x, gridDim.x), o0 = tile % mt * S::BM, i0 = tile / mt * S::BN;
    const int64_t t0 = (int64_t)blockIdx.y * piece, t1 = min(tokens, t0 + piece);
    const int groups = (in + KT_ACT8_GROUP - 1) / KT_ACT8_GROUP, wide = groups * KT_ACT8_GROUP;

    // What a lane has on its way: rows of one step.
    struct Coming {
        u32x4 a[AC > 0 ? AC : 1], b[BC];
        uint32_t e[BC];
    } coming;
    Feed<T, S::BM, K, S::BLOCK, true> feed(dy + t0 * lddy + o0, lddy, (int)min((int64_t)INT32_MAX, t1 - t0), DMA ? out - o0 : 0);
    // x8: through buffers that end at row t1, whose zeros (q = 0, e = 0) make nothing of what the tile holds past it.  Columns past the last
    // are the next row's or zeros and end in columns of the tile that are not stored.
    int at_b[BC], at_e[BC];
#pragma unroll
    for (int u = 0; u < BC; ++u) {
        const int n = tid + u * S::BLOCK, row = n / (S::BN / 16), c = i0 + n % (S::BN / 16) * 16;
        at_b[u] = !BPART || row < K ? row * wide + c : INT32_MIN;
        at_e[u] = !BPART || row < K ? row * groups + c / KT_ACT8_GROUP : INT32_MIN;
    }
    auto load_b = [&](int64_t t, Coming &x) {
        const int rows = (int)max((int64_t)0, min((int64_t)K, t1 - t));
#pragma unroll
        for (int u = 0; u < BC; ++u) {
            x.b[u] = buffer16(q + t * wide, rows * wide, at_b[u]);
            x.e[u] = buffer1(e + t * groups, rows * groups, at_e[u]);
        }
    };
    // dy through registers: rows at and past t1 and columns past the last are zeros.
    auto load = [&](int64_t t, Coming &x) {
#pragma unroll
        for (int u = 0; u < AC; ++u) {
            const int n = tid + u * S::BLOCK, row = n / (S::BM / V), c = o0 + n % (S::BM / V) * V;
            x.a[u] = t + row < t1 ? ld_chunk(dy + (t + row) * lddy, c, out) : u32x4{0, 0, 0, 0};
        }
        load_b(t, x);
    };
    // The same without a branch, so that the loads stay on their way together: what lies past the last column is the next row's
    // beginning then, in columns that are not stored.  For rows below `last`: all that the tile reads of them lies inside dy and before t1.
    uint32_t at_a[AC > 0 ? AC : 1];
#pragma unroll
    for (int u = 0; u < AC; ++u) {
        const int n = tid + u * S::BLOCK;
        at_a[u] = (uint32_t)(n / (S::BM / V)) * (uint32_t)(lddy * sizeof(T)) + (uint32_t)(o0 + n % (S::BM / V) * V) * (uint32_t)sizeof(T);
    }
    auto load_inside = [&](int64_t t, Coming &x) {
        const char *pa = (const char *)(dy + t * lddy);
#pragma unroll
        for (int u = 0; u < AC; ++u) x.a[u] = ld16(pa + at_a[u]);
        load_b(t, x);
    };
    int64_t last = lddy < 1 << 23 && (tokens - 1) * lddy + out >= o0 + S::BM ? min(t1, ((tokens - 1) * lddy + out - o0 - S::BM) / lddy + 1) : 0;
    if (DMA) last = INT64_MAX / 2;
    // Chunk number `u` of the AC + BC * BU that a lane writes into LDS.
    constexpr int STORES = AC + BC * BU;
    auto store = [&](char *buf, const Coming &x, auto u0) {
        constexpr int u = u0;
        if constexpr (u < AC) {
            const int n = tid + u * S::BLOCK;
            *(u32x4 *)(buf + TA::at(n / (S::BM / V), n % (S::BM / V))) = x.a[u];
        } else {
            constexpr int w = (u - AC) / BU, j = (u - AC) % BU;
            const int n = tid + w * S::BLOCK, row = n / (S::BN / 16), c = n % (S::BN / 16);
            if (BPART && row >= K) return;
            float f[V];
#pragma unroll
            for (int k = 0; k < V / 4; ++k) from_bytes(x.b[w][j * (V / 4) + k], step_of(x.e[w]), f + 4 * k);
            *(u32x4 *)(buf + TA::bytes(K) + TB::at(row, c * BU + j)) = narrow<T>(f);
        }
    };

    f32x16 acc[S::FM][S::FN];
#pragma unroll
    for (int m = 0; m < S::FM; ++m)
#pragma unroll
        for (int n = 0; n < S::FN; ++n) acc[m][n] = f32x16{0};
    const int m0 = wave / S::WN * S::FM * 32, n0 = wave % S::WN * S::FN * 32;

    // One step: the products of `now`, beside them what is coming goes into `next`.
    constexpr int PER = S::FM * S::FN, N = K / 16 * PER, READS = S::FM + S::FN;
    auto step = [&](const char *now, char *next, const Coming &x) {
        const char *ta = now, *tb = now + TA::bytes(K);
        constexpr int SETS = sizeof(T) == 2 ? 2 : 1;        // f32: products of 512 cycles need no reads ahead
        F fa[SETS][S::FM], fb[SETS][S::FN];
        auto read = [&](auto c0, auto r0) {
            constexpr int c = c0, r = r0;
            if constexpr (r < S::FM) fa[c % SETS][r] = load_t<T, S::BM>(ta, c, m0 + 32 * r);
            else fb[c % SETS][r - S::FM] = load_t<T, S::BN>(tb, c, n0 + 32 * (r - S::FM));
        };
        auto product = [&](auto n1) {
            constexpr int n = n1, c = n / PER, i = n % PER;
            if constexpr (SETS == 1 && c && i == 0) span<0, READS>([&](auto r) { read(std::integral_constant<int, c>(), r); });
            mma(acc[i / S::FN][i % S::FN], fa[c % SETS][i / S::FN], fb[c % SETS][i % S::FN]);
            if constexpr (SETS == 2 && c + 1 < K / 16)
                span<i * READS / PER, (i + 1) * READS / PER>([&](auto r) { read(std::integral_constant<int, c + 1>(), r); });
            // late among the products: what is coming has had longer to arrive.  Under DMA the wait for x8 is one for dy's tile too, which
            // was started after it: the last quarter (16384 x 2048 x 8192 bf16 493 -> 476 us); else the second half (65 us of 4099 x 1001 x
            // 4004; the last quarter 69).
            constexpr int late = DMA ? N * 3 / 4 : N / 2, from = n < late ? 0 : (n - late) * STORES / (N - late), to = n < late ? 0 : (n - late + 1) * STORES / (N - late);
            span<from, to>([&](auto u) { store(next, x, u); });
            __builtin_amdgcn_sched_barrier(0);
        };
        span<0, READS>([&](auto r) { read(std::integral_constant<int, 0>(), r); });
        __builtin_amdgcn_sched_barrier(0);
        span<0, N>(product);
    };

    // in pairs of steps: rows past the last are zeros
    auto half = [&](int64_t t, char *now, char *next, auto bring) {
        if (DMA) feed.start(next, (int)(t - t0) + K);
        step(now, next, coming);
        bring(t + 2 * K, coming);
        if (DMA) arrived<2 * BC>();                         // the loads of the line before may still be on their way
        __syncthreads();
    };
    auto pair = [&](int64_t t, auto bring) {
        half(t, lds, lds + HALF, bring);
        half(t + K, lds + HALF, lds, bring);
    };
    int64_t t = t0;
    if (t < t1) {
        if (DMA) feed.start(lds, 0);
        load(t0, coming);
        span<0, STORES>([&](auto u) { store(lds, coming, u); });
        load(t0 + K, coming);
        if (DMA) arrived();
        __syncthreads();
    }
    for (; t < t1 && t + 4 * K <= last; t += 2 * K) pair(t, load_inside);
    if (!DMA)
        for (; t < t1; t += 2 * K) pair(t, load);
    if (PIECES) dw += (int64_t)blockIdx.y * out * lddw;
    const int col = lane & 31, h = lane >> 5;
#pragma unroll
    for (int m = 0; m < S::FM; ++m)
#pragma unroll
        for (int n = 0; n < S::FN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int o = o0 + m0 + 32 * m + r % 4 + 8 * (r / 4) + 4 * h, i = i0 + n0 + 32 * n + col;
                if (o < out && i < in) dw[o * lddw + i] = (G)acc[m][n][r];
            }
}

// Sum of the pieces, in their order.
template <typename G>
__global__ __launch_bounds__(256) void kt_weight_grad_sum_kernel(const float *parts, int pieces, int out, int in, int ld, G *dw,
                                                                 int64_t lddw)
{
    const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (c >= in) return;
    const int64_t size = (int64_t)out * ld;
    for (int o = blockIdx.y; o < out; o += gridDim.y) {
        f32x4 s = *(const f32x4 *)(parts + (int64_t)o * ld + c);
        for (int p = 1; p < pieces; ++p) s += *(const f32x4 *)(parts + p * size + (int64_t)o * ld + c);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < in) dw[o * lddw + c + j] = (G)s[j];
    }
}

// How a product is cut: tile side, pieces of t, rows in a piece.  Both sides of each bound, in us, bf16 with 16 384 tokens where not said:
//  - the largest side that makes 192 tiles: 6144 x 2048 (192 tiles of 256) 433 whole, in tiles of 128 547; 1024 x 8192 (128 tiles of 256)
//    401 whole, in tiles of 128 302.  f32: 2048 x 2048 of 6 304 tokens 475 in tiles of 128, 480 in tiles of 64; 768 x 2304 (108 tiles of 128)
//    471, in tiles of 64 273.
//  - pieces below 256 tiles, about two workgroups to a CU: 768 x 768 (144 tiles of 64) 162 whole, 87 in two, 63 in three.
//  - 256 tokens to a piece: 768 x 768 of 300 tokens 5.8 whole, 9.0 in two; of 1 024 tokens 13.2 and 12.6 (of 512 the rule loses: 6.6 and 9.8).
//  - 16 pieces: 96 x 130 (6 tiles) 26 in eight, 19 in sixteen.
// The rule does not count the rounds in which workgroups fill the chip, and loses where they fill it badly: 192 to 255 tiles of 256 are cut in
// two (one workgroup to a CU, so 384 take two rounds: 6144 x 2048 470, whole 433); 2048 x 2048 (256 tiles of 128) stays whole at 243, as 64
// tiles of 256 in four pieces it takes 151; 4099 x 1001 x 4004 67, in four pieces of tiles of 256 57.
struct Cut {
    int side, pieces;
    int64_t piece;
};
Cut cut(kt_dtype dt, int64_t tokens, int64_t out, int64_t in)
{
    const int k = dt == KT_F32 ? 32 : 64;
    auto tiles = [&](int64_t s) { return ((out + s - 1) / s) * ((in + s - 1) / s); };
    Cut c{dt == KT_BF16 && tiles(256) >= 192 ? 256 : tiles(128) >= 192 ? 128 : 64, 1, tokens};
    const int64_t n = tiles(c.side);
    if (n < 256) {
        int64_t p = 512 / n, most = tokens / 256;
        if (p > most) p = most;
        if (p > 16) p = 16;
        if (p > 1) {
            c.piece = ((tokens + p - 1) / p + k - 1) / k * k;
            c.pieces = (int)((tokens + c.piece - 1) / c.piece);
        }
    }
    return c;
}
int64_t part_ld(int64_t in) { return (in + 3) / 4 * 4; }

template <typename T, typename S, typename G, bool PIECES, bool DMA>
int go(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens, int out, int in,
       const Cut &c, hipStream_t s)
{
    const int mt = (out + S::BM - 1) / S::BM, nt = (in + S::BN - 1) / S::BN;
    constexpr int LDS = 2 * (Tile<T, S::BM>::bytes(S::template K<T, DMA>) + Tile<T, S::BN>::bytes(S::template K<T, DMA>));
    if (LDS > 65536) {
        const hipError_t e1 = hipFuncSetAttribute((const void *)kt_weight_grad_kernel<T, S, G, PIECES, DMA>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e1 != hipSuccess) return (int)e1;
    }
    kt_weight_grad_kernel<T, S, G, PIECES, DMA><<<dim3((unsigned)mt * nt, c.pieces), S::BLOCK, LDS, s>>>(dy, lddy, q, e, dw, lddw, tokens, out, in, mt, c.piece);
    return (int)hipGetLastError();
}

template <typename T, typename G, bool PIECES, bool DMA>
int by_side(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens, int out, int in,
            const Cut &c, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) {
        if (c.side == 256) return go<T, Big, G, PIECES, DMA>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    }
    if (c.side == 128) return go<T, Mid, G, PIECES, DMA>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    return go<T, Small, G, PIECES, DMA>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
}
template <typename T, typename G, bool PIECES>
int by_rows(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens, int out, int in,
            const Cut &c, hipStream_t s)
{
    constexpr int64_t TO = 16 / sizeof(T);
    if (reinterpret_cast<uintptr_t>(dy) % 16 == 0 && lddy % TO == 0 && out % TO == 0 && lddy * (int64_t)sizeof(T) < 1 << 24 && c.piece < 1 << 30)
        return by_side<T, G, PIECES, true>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    return by_side<T, G, PIECES, false>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
}

template <typename T, typename G>
int weight_grad(kt_dtype dt, const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens,
                int out, int in, float *ws, hipStream_t s)
{
    const Cut c = cut(dt, tokens, out, in);
    if (c.pieces == 1) return by_rows<T, G, false>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    const int ld = (int)part_ld(in);
    const int err = by_rows<T, float, true>(dy, lddy, q, e, ws, ld, tokens, out, in, c, s);
    if (err) return err;
    kt_weight_grad_sum_kernel<G><<<dim3((ld / 4 + 255) / 256, out < 65535 ? out : 65535), 256, 0, s>>>(ws, c.pieces, out, in, ld, dw, lddw);
    return (int)hipGetLastError();
}

}  // namespace

int64_t kt_weight_grad_ws(kt_dtype dt, int64_t tokens, int64_t out, int64_t in)
{
    const Cut c = cut(dt, tokens, out, in);
    return c.pieces == 1 ? 0 : c.pieces * out * part_ld(in) * (int64_t)sizeof(float);
}

int kt_launch_weight_grad(kt_dtype dt, kt_dtype gdt, int64_t tokens, int out, int in, const void *dy, int64_t lddy,
                          const int8_t *q, const uint8_t *e, void *dw, int64_t lddw, float *ws, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dt == KT_F32) {
        if (gdt == KT_F32) return weight_grad(dt, (const float *)dy, lddy, q, e, (float *)dw, lddw, tokens, out, in, ws, s);
        return weight_grad(dt, (const float *)dy, lddy, q, e, (bf16 *)dw, lddw, tokens, out, in, ws, s);
    }
    if (gdt == KT_F32) return weight_grad(dt, (const bf16 *)dy, lddy, q, e, (float *)dw, lddw, tokens, out, in, ws, s);
    return weight_grad(dt, (const bf16 *)dy, lddy, q, e, (bf16 *)dw, lddw, tokens, out, in, ws, s);
}
