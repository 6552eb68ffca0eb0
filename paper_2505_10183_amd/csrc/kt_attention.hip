// Attention, forward and backward.
//
// All products run on the matrix cores (kt_mfma.h), in the types of the tensors; scores, softmax statistics and sums are
// binary32.  A workgroup is four wavefronts.
//
// Forward and dq: a wavefront owns 32 queries, one per lane and half; tiles of keys pass through LDS.  The scores are
// made transposed, S^T[key][query] = K Q^T, so that a lane holds 16 keys of its own query in registers: maximum and sum of
// the softmax are register operations and one exchange between the two halves, and the probabilities, converted, already are
// the operand of the next product, O^T[d][query] = V^T P^T (dq: K^T dS^T).
//
// dk and dv: a wavefront owns 32 keys; tiles of queries pass through LDS.  S[query][key] = Q K^T puts 16 queries of a lane's key
// into registers, and P and dS are the operands of dV^T[d][key] = dO^T P and dK^T[d][key] = Q^T dS.
// The backward pass computes S and dP twice (7 products instead of 5), in exchange for no atomics on dq, no binary32 copy of
// it in memory, and sums whose order is fixed.
//
// Rounding of P and dS to bf16 is that of the operands of the products (the softmax's sum takes P before it).
//
// Measured, and what bounds it: the matrix cores and the softmax's vector work, which only partly run side by side; LDS is busy
// under 30 % of the cycles and memory idle.  Passes are timed by events among others; single kernels in a kernel trace, under which the long
// ones run up to 10 % longer than in such passes.  bf16, 128 wide, 8 x 2048 causal, 16 heads, backward 580 to 605 us a pass; in the trace
// dq 232 (0.89 PFLOP/s, matrix cores busy 52 % of the cycles), dk and dv 410 (0.67, 36 %: 480 registers leave one wavefront to a SIMD, and
// nothing covers its waits).  Forward, 2 x 8191 causal, 16 heads on 4, one sequence of any length: 415 to 490 us with its length, 55 %.
// f32: eight matrix instructions of 64 cycles to a fragment; 32 x 197, 12 heads, 64 wide, backward 206 to 209 us: dq 82, 74 % busy, dk and
// dv 136, 60 %; the eighth wavefront of 197 keys has no work.
//
// Registers spilled to memory (one wavefront or two to a SIMD, see __launch_bounds__): bf16, 128 wide, off 16 bytes forward 42 and dq 790 (8 x
// 2048 causal, 16 heads, rows 129 apart: forward 350 us for 184, backward 1 460 for 600); f32, 128 wide dk and dv 63, off 16 bytes 215.
// One workgroup to 128 queries (dk and dv: keys) of a head whatever their number: 8 heads of 4 096 queries on one key head of 4 096 keys
// are 32 workgroups of dk and dv, backward 980 us; 1 query of 16 heads on 8 192 keys 134 us forward.
#include "kt_mfma.h"

namespace {

constexpr int WAVES = 4, BLOCK = WAVES * 64, OWN = WAVES * 32;      // rows that a workgroup owns
static_assert(BLOCK == KT_ATTENTION_BLOCK && OWN == KT_ATTENTION_OWN, "the host counts workgroups");
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float NEVER = -__builtin_huge_valf();

// Rows of a tile that passes through LDS.
template <typename T> constexpr int ROWS = sizeof(T) == 2 ? 64 : 32;

template <typename T> struct View {
    T *p;
    int64_t batch, token, head;
    __device__ __forceinline__ T *at(int64_t b, int64_t h) const { return p + b * batch + h * head; }
};
template <typename T> struct Args {
    View<T> q, k, v, o, d_o, dq, dk, dv;
    float *lse, *delta;
    const int32_t *k_lens;
    int nq, nk, heads, kv_heads, dim, causal;
    float scale;
    __device__ __forceinline__ int keys(int b) const { return k_lens ? max(0, min(nk, k_lens[b])) : nk; }
};

// A wavefront's 32 rows from row0 on, one per lane and half, as fragments along them: fragment c is elements 16 c + 8 h .. + 7;
// zeros at and past dim and for rows at and past `end`, which are not read.  DMA (see Feed): through a buffer that ends there, without
// a branch, so that all loads of a workgroup's start are on their way together.
template <typename T, int D, bool DMA>
__device__ __forceinline__ void row_frags(typename Frag<T>::type (&f)[D / 16], const T *p, int64_t stride, int row0, int end, int dim)
{
    const int lane = threadIdx.x & 63, row = lane & 31, h = lane >> 5;
    constexpr int PARTS = 8 / VE<T>;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        u32x4 v[PARTS];
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
            const int d = 16 * c + 8 * h + k * VE<T>;
            if constexpr (DMA) {
                const int rows = min(32, end - row0);
                const int bytes = rows > 0 ? ((rows - 1) * (int)stride + dim) * (int)sizeof(T) : 0;
                v[k] = buffer16(p + row0 * stride, bytes, d < dim ? (row * (int)stride + d) * (int)sizeof(T) : INT32_MIN);
            } else {
                v[k] = row0 + row < end ? ld_chunk(p + (row0 + row) * stride, d, dim) : u32x4{0, 0, 0, 0};
            }
        }
        if constexpr (PARTS == 1) {
            f[c] = __builtin_bit_cast(typename Frag<T>::type, v[0]);
        } else {
            f[c] = __builtin_shufflevector(__builtin_bit_cast(f32x4, v[0]), __builtin_bit_cast(f32x4, v[1]), 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
}

// N products one after another.  Product i takes the fragment that load(i) reads from LDS; reads run AHEAD products before
// their use, and what use(i, fragment) computes beside its product stays beside it: nothing moves across a step.  Left to itself the
// compiler reads each fragment right before its product, and puts all vector work between the products.
template <typename T, int AHEAD, typename L, typename U, int... I>
__device__ __forceinline__ void stream(L load, U use, std::integer_sequence<int, I...>)
{
    constexpr int N = sizeof...(I);
    typename Frag<T>::type f[AHEAD];
    auto first = [&](auto i) {
        if constexpr (i < AHEAD) f[i] = load(i);
    };
    auto step = [&](auto i) {
        use(i, f[i % AHEAD]);
        if constexpr (i + AHEAD < N) f[i % AHEAD] = load(std::integral_constant<int, i + AHEAD>());
        __builtin_amdgcn_sched_barrier(0);
    };
    (first(std::integral_constant<int, I>()), ...);
    __builtin_amdgcn_sched_barrier(0);
    (step(std::integral_constant<int, I>()), ...);
}
template <typename T, int AHEAD, int N, typename L, typename U> __device__ __forceinline__ void stream(L load, U use)
{
    stream<T, AHEAD>(load, use, std::make_integer_sequence<int, N>());
}

__device__ __forceinline__ float other_half(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
    return as_f(threadIdx.x & 32 ? a[0] : a[1]);
}

// Row of register r in a 32 x 32 result, of this lane's half.
__device__ __forceinline__ int row_of(int r) { return r % 4 + 8 * (r / 4) + 4 * ((threadIdx.x & 63) >> 5); }

// A transposed result [d][row] to the row in memory: four adjacent elements at a time.  !any: zeros, whatever the sum holds: weights of 0
// leave it 0 * inf where another row of the tile is not finite.
template <typename T, int D>
__device__ __forceinline__ void store_row(T *row, const f32x16 (&acc)[D / 32], float by, bool any, int dim)
{
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = db * 32 + row_of(4 * i);
            float f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = any ? acc[db][4 * i + j] * by : 0.0f;
            if (d + 4 <= dim) {
                if constexpr (sizeof(T) == 4) {
                    st16(row + d, narrow<float>(f));
                } else {
                    typedef u32x2 u32x2_any __attribute__((aligned(2)));
                    *(u32x2_any *)(row + d) = u32x2{pack2(f[0], f[1]), pack2(f[2], f[3])};
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (d + j < dim) row[d + j] = (T)f[j];
            }
        }
}

// The binary32 row in memory is added to a transposed result.
template <int D> __device__ __forceinline__ void add_row(const float *row, f32x16 (&acc)[D / 32], int dim)
{
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4 v = ld_chunk(row, db * 32 + row_of(4 * i), dim);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[db][4 * i + j] += as_f(v[j]);
        }
}

// Rows of OWN and head of a workgroup.  The last rows of all heads come first: under a causal mask they have the most keys, and the
// short ones fill the end of the launch.  (Head by head on each XCD, so that its L2 holds a head's keys: the long blocks of the last
// heads end late; 8 x 2048 causal, 16 heads of 128: dk and dv 370 -> 427 us.)
struct Place {
    int row0, b, h;
};
__device__ __forceinline__ Place place(int blocks, int heads)
{
    const int per = gridDim.x / blocks, bh = blockIdx.x % per, n = blockIdx.x / per;
    return Place{(blocks - 1 - n) * OWN, bh / heads, bh % heads};
}

template <typename T, int D, bool DMA>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || D == 64 ? 2 : 1) void kt_attention_fwd_kernel(Args<T> a, int blocks)
{
    constexpr int R = ROWS<T>, KB = R / 32, BYTES = Tile<T, D>::bytes(R);
    typedef typename Frag<T>::type F;
    __shared__ __align__(16) char kt0[BYTES], vt0[BYTES], kt1[BYTES], vt1[BYTES];
    const Place at = place(blocks, a.heads);
    const int lane = threadIdx.x & 63, wave = wave_id(), hk = at.h / (a.heads / a.kv_heads);
    const int q = at.row0 + wave * 32 + (lane & 31), off = a.nk - a.nq, len = a.keys(at.b);
    const bool there = q < a.nq;
    // keys [0, mine) are seen by this lane's query, [0, all) by some query of the workgroup
    const int mine = there ? (a.causal ? min(len, max(0, q + off + 1)) : len) : 0;
    const int all = a.causal ? min(len, max(0, min(a.nq, at.row0 + OWN) + off)) : len;
    const T *kp = a.k.at(at.b, hk), *vp = a.v.at(at.b, hk);
    F qf[D / 16];
    row_frags<T, D, DMA>(qf, a.q.at(at.b, at.h), a.q.token, at.row0 + wave * 32, a.nq, a.dim);
    f32x16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{0};
    const float c2 = a.scale * LOG2E;
    float m = NEVER, mc = 0.0f, l = 0.0f;         // maximum that the sums refer to, m * c2, and the sum of this half's keys
    // tiles below seen_by_all need no mask; a wavefront's queries see nothing from `most` on
    const int first = at.row0 + wave * 32, seen_by_all = a.causal ? min(len, max(0, at.row0 + off + 1)) : len;
    const int most = first >= a.nq ? 0 : a.causal ? min(len, max(0, min(a.nq, first + 32) + off)) : len;

    Feed<T, D, R, BLOCK, DMA> ks(kp, a.k.token, all, a.dim), vs(vp, a.v.token, all, a.dim);
    auto step = [&](auto edge, int k0, const char *kt, const char *vt, char *ktn, char *vtn) {
        const bool more = k0 + R < all;
        if (more) {
            ks.start(ktn, k0 + R);
            vs.start(vtn, k0 + R);
        }
        if (!edge || k0 < most) {
            constexpr int AHEAD = sizeof(T) == 2 ? 4 : 2;
            constexpr int NS = KB * D / 16, NO = D / 16;            // products of the scores; of a block of 32 keys with v
            f32x16 s[KB];
            F pf[KB][2];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{0};
            auto weigh = [&](int kb, int r) {           // a score becomes a probability
                s[kb][r] = __builtin_amdgcn_exp2f(__fmaf_rn(s[kb][r], c2, -mc));
                l += s[kb][r];
                if (r % 8 == 7) pf[kb][r / 8] = frag_of<T>(s[kb], r / 8);
            };
            auto load = [&](auto n0) -> F {
                constexpr int n = n0;
                if constexpr (n < NS) return load_r<T, D>(kt, 32 * (n % KB), n / KB);
                constexpr int i = n - NS;
                return load_t<T, D>(vt, 2 * (i / NO) + i % NO / (D / 32), 32 * (i % (D / 32)));
            };
            stream<T, AHEAD, NS + KB * NO>(load, [&](auto n0, const F &f) {
                constexpr int n = n0;
                if constexpr (n == NS) {
                    if constexpr (edge) {
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                            for (int r = 0; r < 16; ++r) s[kb][r] = k0 + 32 * kb + row_of(r) < mine ? s[kb][r] : NEVER;
                    }
                    float top = s[0][0];
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
                    top = fmaxf(top, other_half(top));
                    // the reference moves only when a query's maximum has outgrown it by 2^8: probabilities up to 256 lose
                    // nothing in floating point, and the sums are seldom multiplied
                    if (__any((top - m) * c2 > 8.0f)) {
                        const float next = fmaxf(m, top), by = m == NEVER ? 0.0f : __builtin_amdgcn_exp2f((m - next) * c2);
                        m = next;
                        mc = m == NEVER ? 0.0f : m * c2;
                        l *= by;
#pragma unroll
                        for (int db = 0; db < D / 32; ++db) o[db] *= by;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) weigh(0, r);
                }
                if constexpr (n < NS) {
                    mma(s[n % KB], f, qf[n / KB]);
                } else {
                    constexpr int i = n - NS;
                    mma(o[i % (D / 32)], f, pf[i / NO][i % NO / (D / 32)]);
                    if constexpr (KB > 1 && i < NO) {       // the second block's beside the first block's products
#pragma unroll
                        for (int k = 0; k < 16 / NO; ++k) weigh(1, i * (16 / NO) + k);
                    }
                }
            });
        }
        if (more) {
            ks.finish(ktn);
            vs.finish(vtn);
        }
        arrived();
        __syncthreads();
    };
    if (all > 0) {
        ks.start(kt0, 0);
        vs.start(vt0, 0);
        ks.finish(kt0);
        vs.finish(vt0);
    }
    arrived();
    __syncthreads();
    int k0 = 0;
    for (; k0 + 2 * R <= seen_by_all; k0 += 2 * R) {
        step(std::false_type(), k0, kt0, vt0, kt1, vt1);
        step(std::false_type(), k0 + R, kt1, vt1, kt0, vt0);
    }
    for (; k0 < all; k0 += 2 * R) {
        step(std::true_type(), k0, kt0, vt0, kt1, vt1);
        if (k0 + R < all) step(std::true_type(), k0 + R, kt1, vt1, kt0, vt0);
    }
    if (!there) return;
    l += other_half(l);
    store_row<T, D>(a.o.at(at.b, at.h) + q * a.o.token, o, l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l, mine > 0, a.dim);
    if (a.lse && lane < 32) a.lse[((int64_t)at.b * a.heads + at.h) * a.nq + q] = l == 0.0f ? NEVER : (mc + __log2f(l)) * LN2;
}

// What exp2 subtracts from the scaled score of a query, from its log-sum-exp; a query without keys gets probability 0 for all.
__device__ __forceinline__ float reference(float lse) { return lse == NEVER ? -NEVER : lse * LOG2E; }

template <typename T, int D, bool DMA>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || D == 64 ? 2 : 1) void kt_attention_dq_kernel(Args<T> a, int blocks)
{
    constexpr int R = ROWS<T>, KB = R / 32, BYTES = Tile<T, D>::bytes(R);
    typedef typename Frag<T>::type F;
    __shared__ __align__(16) char kt0[BYTES], vt0[BYTES], kt1[BYTES], vt1[BYTES];
    const Place at = place(blocks, a.heads);
    const int lane = threadIdx.x & 63, wave = wave_id(), hk = at.h / (a.heads / a.kv_heads);
    const int q = at.row0 + wave * 32 + (lane & 31), off = a.nk - a.nq, len = a.keys(at.b);
    const bool there = q < a.nq;
    const int mine = there ? (a.causal ? min(len, max(0, q + off + 1)) : len) : 0;
    const int all = a.causal ? min(len, max(0, min(a.nq, at.row0 + OWN) + off)) : len;
    const int first = at.row0 + wave * 32, seen_by_all = a.causal ? min(len, max(0, at.row0 + off + 1)) : len;
    const int most = first >= a.nq ? 0 : a.causal ? min(len, max(0, min(a.nq, first + 32) + off)) : len;
    const T *kp = a.k.at(at.b, hk), *vp = a.v.at(at.b, hk);
    Feed<T, D, R, BLOCK, DMA> ks(kp, a.k.token, all, a.dim), vs(vp, a.v.token, all, a.dim);
    if (all > 0) {
        ks.start(kt0, 0);
        vs.start(vt0, 0);
    }

    F qf[D / 16], df[D / 16];
    float delta = 0.0f;
    {
        F of[D / 16];
        row_frags<T, D, DMA>(qf, a.q.at(at.b, at.h), a.q.token, first, a.nq, a.dim);
        row_frags<T, D, DMA>(df, a.d_o.at(at.b, at.h), a.d_o.token, first, a.nq, a.dim);
        row_frags<T, D, DMA>(of, a.o.at(at.b, at.h), a.o.token, first, a.nq, a.dim);
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta = __fmaf_rn((float)df[c][j], (float)of[c][j], delta);
        delta += other_half(delta);
    }
    const int64_t stat = ((int64_t)at.b * a.heads + at.h) * a.nq + q;
    if (there && lane < 32) a.delta[stat] = delta;
    const float c2 = a.scale * LOG2E, ref = there ? reference(a.lse[stat]) : -NEVER;
    f32x16 dq[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dq[db] = f32x16{0};

    auto step = [&](auto edge, int k0, const char *kt, const char *vt, char *ktn, char *vtn) {
        const bool more = k0 + R < all;
        if (more) {
            ks.start(ktn, k0 + R);
            vs.start(vtn, k0 + R);
        }
        if (!edge || k0 < most) {
            constexpr int AHEAD = sizeof(T) == 2 ? 6 : 2;
            constexpr int NS = 2 * D / 16, NO = D / 16;             // products of a block of 32 keys: s and dp; dq
            f32x16 s, dp;
            F sf[2];
            auto load = [&](auto n0) -> F {
                constexpr int n = n0, kb = n / (NS + NO), i = n % (NS + NO);
                if constexpr (i < NS) return load_r<T, D>(i % 2 ? vt : kt, 32 * kb, i / 2);
                else return load_t<T, D>(kt, 2 * kb + (i - NS) / (D / 32), 32 * ((i - NS) % (D / 32)));
            };
            stream<T, AHEAD, KB * (NS + NO)>(load, [&](auto n0, const F &f) {
                constexpr int n = n0, kb = n / (NS + NO), i = n % (NS + NO);
                if constexpr (i == 0) s = dp = f32x16{0};
                if constexpr (i == NS) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(__fmaf_rn(s[r], c2, -ref));
                        s[r] = p * (dp[r] - delta);
                        if constexpr (edge) s[r] = k0 + 32 * kb + row_of(r) < mine ? s[r] : 0.0f;
                    }
                    sf[0] = frag_of<T>(s, 0);
                    sf[1] = frag_of<T>(s, 1);
                }
                if constexpr (i < NS) {
                    if constexpr (i % 2) mma(dp, f, df[i / 2]);
                    else mma(s, f, qf[i / 2]);
                } else {
                    mma(dq[(i - NS) % (D / 32)], f, sf[(i - NS) / (D / 32)]);
                }
            });
        }
        if (more) {
            ks.finish(ktn);
            vs.finish(vtn);
        }
        arrived();
        __syncthreads();
    };
    if (all > 0) {
        ks.finish(kt0);
        vs.finish(vt0);
    }
    arrived();
    __syncthreads();
    int k0 = 0;
    for (; k0 + 2 * R <= seen_by_all; k0 += 2 * R) {
        step(std::false_type(), k0, kt0, vt0, kt1, vt1);
        step(std::false_type(), k0 + R, kt1, vt1, kt0, vt0);
    }
    for (; k0 < all; k0 += 2 * R) {
        step(std::true_type(), k0, kt0, vt0, kt1, vt1);
        if (k0 + R < all) step(std::true_type(), k0 + R, kt1, vt1, kt0, vt0);
    }
    if (there) store_row<T, D>(a.dq.at(at.b, at.h) + q * a.dq.token, dq, a.scale, mine > 0, a.dim);
}

// Tiles of queries after which f32 puts its sums into the rows of dk and dv in memory, which this workgroup alone writes, and begins
// new ones: 512 queries.  One chain over all of them loses digits that the type has: 4 heads of 4 096 queries to a key head stood
// 2.4e-6 from the formulas in norm, in pieces 8e-7.  It costs 3 % of the backward pass 64 wide (4 x 1024, 12 heads, 473 -> 485 us)
// and 5 to 8 % 128 wide (951 -> 994), where the rows' way through memory takes registers that the steps need.  bf16 rounds to
// 2^-8 at the end.
constexpr int PIECE = 16;

// One wavefront to a SIMD: f32 of 64 held to 256 registers for two of them spills 39 (32 x 197, 12 heads: backward 206 -> 227 us).
template <typename T, int D, bool DMA>
__global__ __launch_bounds__(BLOCK, 1) void kt_attention_dkv_kernel(Args<T> a, int blocks)
{
    constexpr int R = ROWS<T>, QB = R / 32, BYTES = Tile<T, D>::bytes(R);
    typedef typename Frag<T>::type F;
    __shared__ __align__(16) char qt0[BYTES], dt0[BYTES], qt1[BYTES], dt1[BYTES];
    __shared__ __align__(16) float stat0[2 * R], stat1[2 * R];
    const int per = gridDim.x / blocks, bh = blockIdx.x % per, k0 = blockIdx.x / per * OWN;     // the first keys have the most queries
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads, group = a.heads / a.kv_heads;
    const int lane = threadIdx.x & 63, wave = wave_id(), off = a.nk - a.nq, len = a.keys(b);
    const int first = k0 + wave * 32, key = first + (lane & 31);
    const bool there = key < len;                   // seen by some query; others get gradient 0 (key < nk)
    F kf[D / 16], vf[D / 16];
    row_frags<T, D, DMA>(kf, a.k.at(b, hk), a.k.token, first, len, a.dim);
    row_frags<T, D, DMA>(vf, a.v.at(b, hk), a.v.token, first, len, a.dim);
    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[db] = dv[db] = f32x16{0};
    const float c2 = a.scale * LOG2E;
    // queries [from, nq) see a key of the workgroup, those from `mine0` on one of this wavefront; those from `full` on see all keys of
    // the workgroup, and their tiles need no mask.  A head's tiles are taken in pairs: an odd one more is all zeros.
    const int from = k0 >= len ? a.nq : a.causal ? max(0, k0 - off) / R * R : 0;
    const int mine0 = first >= len ? a.nq : a.causal ? max(0, first - off) : 0;
    const int mine = a.causal ? key - off : 0;      // first query that sees this lane's key
    const int full = k0 + OWN > len ? a.nq : a.causal ? max(0, k0 + OWN - 1 - off) : 0;
    const int upto = from + (a.nq - from + 2 * R - 1) / (2 * R) * (2 * R);
    const int mid = from + (max(0, full - from) + 2 * R - 1) / (2 * R) * (2 * R);

    Feed<T, D, R, BLOCK, DMA> qs(a.q.at(b, hk * group), a.q.token, a.nq, a.dim), ds(a.d_o.at(b, hk * group), a.d_o.token, a.nq, a.dim);
    float stat;
    const float *stats = threadIdx.x < R ? a.lse : a.delta;
    stats += ((int64_t)b * a.heads + hk * group) * a.nq;
    auto start = [&](int q0, char *qt, char *dt) {
        qs.start(qt, q0);
        ds.start(dt, q0);
        if (threadIdx.x < 2 * R) {
            const int q = q0 + threadIdx.x % R;
            stat = q < a.nq ? stats[q] : threadIdx.x < R ? NEVER : 0.0f;
        }
    };
    auto finish = [&](char *qt, char *dt, float *st) {
        qs.finish(qt);
        ds.finish(dt);
        if (threadIdx.x < 2 * R) st[threadIdx.x] = threadIdx.x < R ? reference(stat) : stat;
    };
    int g = 0, q0 = from;
    auto step = [&](auto edge, const char *qt, const char *dt, const float *refs, char *qtn, char *dtn, float *refsn) {
        const float *deltas = refs + R;
        int nq0 = q0 + R;
        if (nq0 >= upto && g + 1 < group) {         // the next head that shares these keys
            ++g;
            nq0 = from;
            qs.p += a.q.head;
            ds.p += a.d_o.head;
            stats += a.nq;
        }
        const bool more = nq0 < upto;
        if (more) start(nq0, qtn, dtn);
        if (!edge || q0 + R > mine0) {
            constexpr int AHEAD = sizeof(T) == 2 ? 6 : 2;
            constexpr int NS = 2 * D / 16, NO = 4 * D / 32;         // products of a block of 32 queries: s and dp; dv and dk
            f32x16 s[QB], dp[QB];
            f32x4 ref[QB][4], delta[QB][4];
            F pf[QB][2], sf[QB][2];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                s[qb] = dp[qb] = f32x16{0};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ref[qb][i] = *(const f32x4 *)(refs + 32 * qb + row_of(4 * i));
                    delta[qb][i] = *(const f32x4 *)(deltas + 32 * qb + row_of(4 * i));
                }
            }
            auto weigh = [&](int qb, int r) {
                float p = __builtin_amdgcn_exp2f(__fmaf_rn(s[qb][r], c2, -ref[qb][r / 4][r % 4]));
                float d = p * (dp[qb][r] - delta[qb][r / 4][r % 4]);
                if constexpr (edge) {               // after the product, which may be 0 * inf
                    const bool sees = there && q0 + 32 * qb + row_of(r) >= mine;
                    p = sees ? p : 0.0f;
                    d = sees ? d : 0.0f;
                }
                dp[qb][r] = d;
                s[qb][r] = p;
                if (r % 8 == 7) {
                    pf[qb][r / 8] = frag_of<T>(s[qb], r / 8);
                    sf[qb][r / 8] = frag_of<T>(dp[qb], r / 8);
                }
            };
            auto load = [&](auto n0) -> F {
                constexpr int n = n0;
                if constexpr (n < QB * NS) return load_r<T, D>(n % 2 ? dt : qt, 32 * (n / NS), n % NS / 2);
                constexpr int i = n - QB * NS;
                return load_t<T, D>(i % 2 ? qt : dt, 2 * (i / NO) + i % NO / (NO / 2), 32 * (i / 2 % (D / 32)));
            };
            stream<T, AHEAD, QB * (NS + NO)>(load, [&](auto n0, const F &f) {
                constexpr int n = n0;
                if constexpr (QB == 1 && n == NS) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) weigh(0, r);
                }
                if constexpr (n < QB * NS) {
                    constexpr int qb = n / NS;
                    if constexpr (n % 2) mma(dp[qb], f, vf[n % NS / 2]);
                    else mma(s[qb], f, kf[n % NS / 2]);
                    if constexpr (qb == 1) {                // the first block's beside the second block's products
#pragma unroll
                        for (int k = 0; k < 16 / NS; ++k) weigh(0, n % NS * (16 / NS) + k);
                    }
                } else {
                    constexpr int i = n - QB * NS, qb = i / NO, c = i % NO / (NO / 2), db = i / 2 % (D / 32);
                    if constexpr (i % 2) mma(dk[db], f, sf[qb][c]);
                    else mma(dv[db], f, pf[qb][c]);
                    if constexpr (QB > 1 && i < NO) {
#pragma unroll
                        for (int k = 0; k < 16 / NO; ++k) weigh(1, i * (16 / NO) + k);
                    }
                }
            });
        }
        if (more) finish(qtn, dtn, refsn);
        arrived();
        __syncthreads();
        q0 = nq0;
    };
    if (q0 < a.nq) {
        start(q0, qt0, dt0);
        finish(qt0, dt0, stat0);
    }
    arrived();
    __syncthreads();
    T *dk_row = a.dk.at(b, hk) + key * a.dk.token, *dv_row = a.dv.at(b, hk) + key * a.dv.token;
    constexpr bool PIECES = sizeof(T) == 4;
    int left = PIECE;                               // tiles until the sums are put into memory
    bool begun = false;                             // the rows in memory hold the sums of earlier pieces
    while (q0 < upto) {
        while (q0 < mid && q0 < upto && left) {     // of the last head q0 ends at upto, of the others at from again
            step(std::true_type(), qt0, dt0, stat0, qt1, dt1, stat1);
            step(std::true_type(), qt1, dt1, stat1, qt0, dt0, stat0);
            if constexpr (PIECES) left -= 2;
        }
        while (q0 >= mid && q0 < upto && left) {
            step(std::false_type(), qt0, dt0, stat0, qt1, dt1, stat1);
            step(std::false_type(), qt1, dt1, stat1, qt0, dt0, stat0);
            if constexpr (PIECES) left -= 2;
        }
        if constexpr (PIECES) {
            if (left || q0 >= upto) continue;
            if (key < a.nk) {
                if (begun) {
                    add_row<D>(dk_row, dk, a.dim);
                    add_row<D>(dv_row, dv, a.dim);
                }
                store_row<T, D>(dk_row, dk, 1.0f, there, a.dim);
                store_row<T, D>(dv_row, dv, 1.0f, there, a.dim);
            }
#pragma unroll
            for (int db = 0; db < D / 32; ++db) dk[db] = dv[db] = f32x16{0};
            begun = true;
            left = PIECE;
        }
    }
    if (key < a.nk) {
        if constexpr (PIECES) {
            if (begun) {
                add_row<D>(dk_row, dk, a.dim);
                add_row<D>(dv_row, dv, a.dim);
            }
        }
        store_row<T, D>(dk_row, dk, a.scale, there, a.dim);
        store_row<T, D>(dv_row, dv, 1.0f, there, a.dim);
    }
}

template <typename T> View<T> view(const kt_heads *h)
{
    return h ? View<T>{(T *)h->data, h->batch, h->token, h->head} : View<T>{nullptr, 0, 0, 0};
}

template <typename T> Args<T> args(const kt_attention *a)
{
    Args<T> r{};
    r.k_lens = a->k_lens;
    r.nq = (int)a->nq;
    r.nk = (int)a->nk;
    r.heads = (int)a->heads;
    r.kv_heads = (int)a->kv_heads;
    r.dim = (int)a->dim;
    r.causal = a->causal != 0;
    r.scale = a->scale;
    return r;
}

// Whether tiles of these rows can be brought by DMA (Feed).
template <typename T> bool dma(const View<T> &v, int dim)
{
    const int64_t to = 16 / sizeof(T);
    return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.batch % to == 0 && v.token % to == 0 && v.head % to == 0 && dim % to == 0 &&
           v.token * (int64_t)sizeof(T) < (1 << 24);
}

template <typename T, int D, bool DMA> int fwd(const kt_attention *a, const Args<T> &r, hipStream_t s)
{
    const int blocks = (r.nq + OWN - 1) / OWN;
    kt_attention_fwd_kernel<T, D, DMA><<<(unsigned)(a->batch * a->heads * blocks), BLOCK, 0, s>>>(r, blocks);
    return (int)hipGetLastError();
}

template <typename T, int D, bool DMA> int bwd(const kt_attention *a, const Args<T> &r, hipStream_t s)
{
    const int qb = (r.nq + OWN - 1) / OWN, kb = (r.nk + OWN - 1) / OWN;
    if (qb) {
        kt_attention_dq_kernel<T, D, DMA><<<(unsigned)(a->batch * a->heads * qb), BLOCK, 0, s>>>(r, qb);
        const int e = (int)hipGetLastError();
        if (e) return e;
    }
    if (!kb) return 0;
    kt_attention_dkv_kernel<T, D, DMA><<<(unsigned)(a->batch * a->kv_heads * kb), BLOCK, 0, s>>>(r, kb);
    return (int)hipGetLastError();
}

template <typename T>
int forward(const kt_attention *a, const kt_heads *q, const kt_heads *k, const kt_heads *v, const kt_heads *o, float *lse, hipStream_t s)
{
    Args<T> r = args<T>(a);
    r.q = view<T>(q);
    r.k = view<T>(k);
    r.v = view<T>(v);
    r.o = view<T>(o);
    r.lse = lse;
    if (dma(r.q, r.dim) && dma(r.k, r.dim) && dma(r.v, r.dim)) return r.dim <= 64 ? fwd<T, 64, true>(a, r, s) : fwd<T, 128, true>(a, r, s);
    return r.dim <= 64 ? fwd<T, 64, false>(a, r, s) : fwd<T, 128, false>(a, r, s);
}

template <typename T>
int backward(const kt_attention *a, const kt_heads *d_o, const kt_heads *q, const kt_heads *k, const kt_heads *v, const kt_heads *o,
             const float *lse, const kt_heads *dq, const kt_heads *dk, const kt_heads *dv, float *ws, hipStream_t s)
{
    Args<T> r = args<T>(a);
    r.q = view<T>(q);
    r.k = view<T>(k);
    r.v = view<T>(v);
    r.o = view<T>(o);
    r.d_o = view<T>(d_o);
    r.dq = view<T>(dq);
    r.dk = view<T>(dk);
    r.dv = view<T>(dv);
    r.lse = const_cast<float *>(lse);
    r.delta = ws;
    if (dma(r.q, r.dim) && dma(r.k, r.dim) && dma(r.v, r.dim) && dma(r.o, r.dim) && dma(r.d_o, r.dim))
        return r.dim <= 64 ? bwd<T, 64, true>(a, r, s) : bwd<T, 128, true>(a, r, s);
    return r.dim <= 64 ? bwd<T, 64, false>(a, r, s) : bwd<T, 128, false>(a, r, s);
}

}  // namespace

int64_t kt_attention_bwd_ws(const kt_attention *a) { return a->batch * a->heads * a->nq * (int64_t)sizeof(float); }

int kt_launch_attention_fwd(const kt_attention *a, const kt_heads *q, const kt_heads *k, const kt_heads *v, const kt_heads *o,
                            float *lse, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    return a->dt == KT_F32 ? forward<float>(a, q, k, v, o, lse, s) : forward<bf16>(a, q, k, v, o, lse, s);
}

int kt_launch_attention_bwd(const kt_attention *a, const kt_heads *d_o, const kt_heads *q, const kt_heads *k, const kt_heads *v,
                            const kt_heads *o, const float *lse, const kt_heads *dq, const kt_heads *dk, const kt_heads *dv,
                            float *ws, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    return a->dt == KT_F32 ? backward<float>(a, d_o, q, k, v, o, lse, dq, dk, dv, ws, s)
                           : backward<bf16>(a, d_o, q, k, v, o, lse, dq, dk, dv, ws, s);
}
