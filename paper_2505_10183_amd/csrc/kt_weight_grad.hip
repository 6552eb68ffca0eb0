// The weight gradient of a linear layer from the 8-bit checkpoint of its input: dw[o][i] = sum_t dy[t][o] x8[t][i].
//
// Both operands run over t along their rows, so both are read across rows from LDS.  A workgroup makes a tile of BM x BN of dw: per
// step, BK rows of dy and of x8 go from memory into registers while the step before is multiplied, x8 is turned into
// dy's type on its way into LDS (exact in bf16: 7 bits and a power of two), and the two halves of LDS take turns, one barrier
// a step.  Where dw has too few tiles for the chip, t is cut into pieces whose sums a second kernel adds in their order.
#include "kt_mfma.h"

namespace {

template <typename T> constexpr int BK = 64 / (int)sizeof(T);          // 32 rows of bf16, 16 of f32

// Tile and wavefronts: WM x WN of them, each FM x FN products of 32 x 32.
template <int WM_, int WN_, int FM_, int FN_> struct Shape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32, BLOCK = WM * WN * 64;
};
typedef Shape<2, 4, 4, 2> Big;       // 256 x 256, 8 wavefronts
typedef Shape<2, 2, 2, 2> Mid;       // 128 x 128, 4
typedef Shape<2, 2, 1, 1> Small;     //  64 x  64, 4

// Tile of a workgroup: those of one XCD (every eighth workgroup) are neighbours, dy's columns first, so that its L2 keeps a
// strip of x8 and all of dy's current rows.
__device__ __forceinline__ int xcd_order(int b, int n)
{
    const int q = n / 8, r = n % 8, x = b % 8;
    return x * q + min(x, r) + b / 8;
}

template <typename T, typename S, typename G, bool PIECES>
__global__ __launch_bounds__(S::BLOCK) void kt_weight_grad_kernel(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e,
                                                                  G *dw, int64_t lddw, int64_t tokens, int out, int in, int mt,
                                                                  int64_t piece)
{
    constexpr int K = BK<T>, V = VE<T>;
    constexpr int AC = K * S::BM / V / S::BLOCK;            // 16-byte chunks of dy that a lane brings
    constexpr int BC = K * S::BN / 16 / S::BLOCK > 0 ? K * S::BN / 16 / S::BLOCK : 1;        // 16 bytes of x8 each
    constexpr bool BPART = K * S::BN / 16 < S::BLOCK;       // the first lanes only
    typedef Tile<T, S::BM> TA;
    typedef Tile<T, S::BN> TB;
    __shared__ __align__(16) char lds[2][TA::bytes(K) + TB::bytes(K)];

    const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
    const int tile = xcd_order(blockIdx.x, gridDim.x), o0 = tile % mt * S::BM, i0 = tile / mt * S::BN;
    const int64_t t0 = (int64_t)blockIdx.y * piece, t1 = min(tokens, t0 + piece);
    const int groups = (in + KT_ACT8_GROUP - 1) / KT_ACT8_GROUP, wide = groups * KT_ACT8_GROUP;

    u32x4 a[AC], b[BC];
    uint32_t eb[BC];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int u = 0; u < AC; ++u) {
            const int n = tid + u * S::BLOCK, row = n / (S::BM / V), c = o0 + n % (S::BM / V) * V;
            a[u] = t + row < t1 ? ld_chunk(dy + (t + row) * lddy, c, out) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < BC; ++u) {
            const int n = tid + u * S::BLOCK, row = n / (S::BN / 16), c = i0 + n % (S::BN / 16) * 16;
            b[u] = u32x4{0, 0, 0, 0};
            eb[u] = 0;
            if ((!BPART || row < K) && t + row < t1 && c < wide) {
                b[u] = *(const u32x4 *)(q + (t + row) * wide + c);
                eb[u] = e[(t + row) * groups + c / KT_ACT8_GROUP];
            }
        }
    };
    auto store = [&](char *buf) {
#pragma unroll
        for (int u = 0; u < AC; ++u) {
            const int n = tid + u * S::BLOCK;
            *(u32x4 *)(buf + TA::at(n / (S::BM / V), n % (S::BM / V))) = a[u];
        }
        char *bb = buf + TA::bytes(K);
#pragma unroll
        for (int u = 0; u < BC; ++u) {
            const int n = tid + u * S::BLOCK, row = n / (S::BN / 16), c = n % (S::BN / 16);
            if (BPART && row >= K) break;
            const float step = step_of(eb[u]);
            float f[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) from_bytes(b[u][j], step, f + 4 * j);
#pragma unroll
            for (int j = 0; j < 16 / V; ++j) *(u32x4 *)(bb + TB::at(row, c * (16 / V) + j)) = narrow<T>(f + j * V);
        }
    };

    f32x16 acc[S::FM][S::FN];
#pragma unroll
    for (int m = 0; m < S::FM; ++m)
#pragma unroll
        for (int n = 0; n < S::FN; ++n) acc[m][n] = f32x16{0};
    const int m0 = wave / S::WN * S::FM * 32, n0 = wave % S::WN * S::FN * 32;

    load(t0);
    store(lds[0]);
    __syncthreads();
    int half = 0;
    for (int64_t t = t0; t < t1; t += K, half ^= 1) {
        const bool more = t + K < t1;
        if (more) load(t + K);
        const char *ta = lds[half], *tb = ta + TA::bytes(K);
#pragma unroll
        for (int c = 0; c < K / 16; ++c) {
            typename Frag<T>::type fa[S::FM], fb[S::FN];
#pragma unroll
            for (int m = 0; m < S::FM; ++m) fa[m] = load_t<T, S::BM>(ta, c, m0 + 32 * m);
#pragma unroll
            for (int n = 0; n < S::FN; ++n) fb[n] = load_t<T, S::BN>(tb, c, n0 + 32 * n);
#pragma unroll
            for (int m = 0; m < S::FM; ++m)
#pragma unroll
                for (int n = 0; n < S::FN; ++n) mma(acc[m][n], fa[m], fb[n]);
        }
        if (more) store(lds[half ^ 1]);
        __syncthreads();
    }
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

// How a product is cut: tile side, pieces of t, rows in a piece.
struct Cut {
    int side, pieces;
    int64_t piece;
};
Cut cut(kt_dtype dt, int64_t tokens, int64_t out, int64_t in)
{
    const int k = dt == KT_F32 ? BK<float> : BK<bf16>;
    auto tiles = [&](int64_t s) { return ((out + s - 1) / s) * ((in + s - 1) / s); };
    Cut c{tiles(256) >= 192 ? 256 : tiles(128) >= 192 ? 128 : 64, 1, tokens};
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

template <typename T, typename S, typename G, bool PIECES>
int go(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens, int out, int in,
       const Cut &c, hipStream_t s)
{
    const int mt = (out + S::BM - 1) / S::BM, nt = (in + S::BN - 1) / S::BN;
    kt_weight_grad_kernel<T, S, G, PIECES><<<dim3((unsigned)mt * nt, c.pieces), S::BLOCK, 0, s>>>(dy, lddy, q, e, dw, lddw, tokens, out, in, mt, c.piece);
    return (int)hipGetLastError();
}

template <typename T, typename G, bool PIECES>
int by_side(const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens, int out, int in,
            const Cut &c, hipStream_t s)
{
    if (c.side == 256) return go<T, Big, G, PIECES>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    if (c.side == 128) return go<T, Mid, G, PIECES>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    return go<T, Small, G, PIECES>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
}

template <typename T, typename G>
int weight_grad(kt_dtype dt, const T *dy, int64_t lddy, const int8_t *q, const uint8_t *e, G *dw, int64_t lddw, int64_t tokens,
                int out, int in, float *ws, hipStream_t s)
{
    const Cut c = cut(dt, tokens, out, in);
    if (c.pieces == 1) return by_side<T, G, false>(dy, lddy, q, e, dw, lddw, tokens, out, in, c, s);
    const int ld = (int)part_ld(in);
    const int err = by_side<T, float, true>(dy, lddy, q, e, ws, ld, tokens, out, in, c, s);
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
