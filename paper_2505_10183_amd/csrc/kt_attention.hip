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
#include "kt_mfma.h"

namespace {

constexpr int WAVES = 4, BLOCK = WAVES * 64, OWN = WAVES * 32;      // rows that a workgroup owns
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

// Fragment c of a row in memory: elements 16 c + 8 h .. + 7, zeros at and past dim and for rows that are not there.
template <typename T> __device__ __forceinline__ typename Frag<T>::type row_frag(const T *row, bool there, int c, int dim)
{
    const int d = 16 * c + 8 * ((threadIdx.x & 63) >> 5);
    if constexpr (sizeof(T) == 2) {
        return __builtin_bit_cast(bf16x8, there ? ld_chunk(row, d, dim) : u32x4{0, 0, 0, 0});
    } else {
        const u32x4 lo = there ? ld_chunk(row, d, dim) : u32x4{0, 0, 0, 0};
        const u32x4 hi = there ? ld_chunk(row, d + 4, dim) : u32x4{0, 0, 0, 0};
        return __builtin_shufflevector(__builtin_bit_cast(f32x4, lo), __builtin_bit_cast(f32x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// A tile of ROWS rows on its way from memory to LDS; rows at and past `end` are zeros and are not read.
template <typename T, int D> struct Stage {
    static constexpr int V = VE<T>, N = ROWS<T> * D / V / BLOCK;
    u32x4 r[N];
    __device__ __forceinline__ void load(const T *p, int64_t stride, int row0, int end, int dim)
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int n = threadIdx.x + u * BLOCK, row = row0 + n / (D / V);
            r[u] = row < end ? ld_chunk(p + row * stride, n % (D / V) * V, dim) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void store(char *tile) const
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int n = threadIdx.x + u * BLOCK;
            *(u32x4 *)(tile + Tile<T, D>::at(n / (D / V), n % (D / V))) = r[u];
        }
    }
};

__device__ __forceinline__ float other_half(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
    return as_f(threadIdx.x & 32 ? a[0] : a[1]);
}

// Row of register r in a 32 x 32 result, of this lane's half.
__device__ __forceinline__ int row_of(int r) { return r % 4 + 8 * (r / 4) + 4 * ((threadIdx.x & 63) >> 5); }

// A transposed result [d][row] to the row in memory: four adjacent elements at a time.
template <typename T, int D> __device__ __forceinline__ void store_row(T *row, const f32x16 (&acc)[D / 32], float by, int dim)
{
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = db * 32 + row_of(4 * i);
            float f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = acc[db][4 * i + j] * by;
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

// Rows of OWN and head of a workgroup.  The last rows come first: under a causal mask they have the most keys, and the short ones
// fill the end of the launch.
struct Place {
    int row0, b, h;
};
__device__ __forceinline__ Place place(int blocks, int heads)
{
    const int bh = blockIdx.x % (gridDim.x / blocks), n = blockIdx.x / (gridDim.x / blocks);
    return Place{(blocks - 1 - n) * OWN, bh / heads, bh % heads};
}

template <typename T, int D>
__global__ __launch_bounds__(BLOCK, 2) void kt_attention_fwd_kernel(Args<T> a, int blocks)
{
    constexpr int R = ROWS<T>, KB = R / 32;
    typedef typename Frag<T>::type F;
    __shared__ __align__(16) char kt[Tile<T, D>::bytes(R)], vt[Tile<T, D>::bytes(R)];
    const Place at = place(blocks, a.heads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, hk = at.h / (a.heads / a.kv_heads);
    const int q = at.row0 + wave * 32 + (lane & 31), off = a.nk - a.nq, len = a.keys(at.b);
    const bool there = q < a.nq;
    // keys [0, mine) are seen by this lane's query, [0, all) by some query of the workgroup
    const int mine = there ? (a.causal ? min(len, max(0, q + off + 1)) : len) : 0;
    const int all = a.causal ? min(len, max(0, min(a.nq, at.row0 + OWN) + off)) : len;
    const T *kp = a.k.at(at.b, hk), *vp = a.v.at(at.b, hk), *qp = a.q.at(at.b, at.h) + q * a.q.token;
    F qf[D / 16];
#pragma unroll
    for (int c = 0; c < D / 16; ++c) qf[c] = row_frag(qp, there, c, a.dim);
    f32x16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{0};
    const float c2 = a.scale * LOG2E;
    float m = NEVER, mc = 0.0f, l = 0.0f;         // maximum that the sums refer to, m * c2, and the sum of this half's keys
    // the fewest and the most keys that a query of this wavefront sees: tiles below the first need no mask
    const int first = at.row0 + wave * 32, least = a.causal ? min(len, max(0, first + off + 1)) : len;
    const int most = first >= a.nq ? 0 : a.causal ? min(len, max(0, min(a.nq, first + 32) + off)) : len;

    Stage<T, D> ks, vs;
    ks.load(kp, a.k.token, 0, all, a.dim);
    vs.load(vp, a.v.token, 0, all, a.dim);
    for (int k0 = 0; k0 < all; k0 += R) {
        ks.store(kt);
        vs.store(vt);
        __syncthreads();
        if (k0 + R < all) {
            ks.load(kp, a.k.token, k0 + R, all, a.dim);
            vs.load(vp, a.v.token, k0 + R, all, a.dim);
        }
        if (k0 < most) {
            f32x16 s[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                s[kb] = f32x16{0};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) mma(s[kb], load_r<T, D>(kt, 32 * kb, c), qf[c]);
            }
            if (k0 + R > least) {
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
            // the reference moves only when a query's maximum has outgrown it by 2^8: probabilities up to 256 lose nothing
            // in floating point, and the sums are seldom multiplied
            if (__any((top - m) * c2 > 8.0f)) {
                const float next = fmaxf(m, top), by = m == NEVER ? 0.0f : __builtin_amdgcn_exp2f((m - next) * c2);
                m = next;
                mc = m == NEVER ? 0.0f : m * c2;
                l *= by;
#pragma unroll
                for (int db = 0; db < D / 32; ++db) o[db] *= by;
            }
            F pf[KB][2];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[kb][r] = __builtin_amdgcn_exp2f(__fmaf_rn(s[kb][r], c2, -mc));
                    l += s[kb][r];
                }
                pf[kb][0] = frag_of<T>(s[kb], 0);
                pf[kb][1] = frag_of<T>(s[kb], 1);
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) mma(o[db], load_t<T, D>(vt, 2 * kb + c, 32 * db), pf[kb][c]);
        }
        __syncthreads();
    }
    if (!there) return;
    l += other_half(l);
    store_row<T, D>(a.o.at(at.b, at.h) + q * a.o.token, o, l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l, a.dim);
    if (a.lse && lane < 32) a.lse[((int64_t)at.b * a.heads + at.h) * a.nq + q] = l == 0.0f ? NEVER : (mc + __log2f(l)) * LN2;
}

// What exp2 subtracts from the scaled score of a query, from its log-sum-exp; a query without keys gets probability 0 for all.
__device__ __forceinline__ float reference(float lse) { return lse == NEVER ? -NEVER : lse * LOG2E; }

template <typename T, int D>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || D == 64 ? 2 : 1) void kt_attention_dq_kernel(Args<T> a, int blocks)
{
    constexpr int R = ROWS<T>, KB = R / 32;
    typedef typename Frag<T>::type F;
    __shared__ __align__(16) char kt[Tile<T, D>::bytes(R)], vt[Tile<T, D>::bytes(R)];
    const Place at = place(blocks, a.heads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, hk = at.h / (a.heads / a.kv_heads);
    const int q = at.row0 + wave * 32 + (lane & 31), off = a.nk - a.nq, len = a.keys(at.b);
    const bool there = q < a.nq;
    const int mine = there ? (a.causal ? min(len, max(0, q + off + 1)) : len) : 0;
    const int all = a.causal ? min(len, max(0, min(a.nq, at.row0 + OWN) + off)) : len;
    const int first = at.row0 + wave * 32, least = a.causal ? min(len, max(0, first + off + 1)) : len;
    const int most = first >= a.nq ? 0 : a.causal ? min(len, max(0, min(a.nq, first + 32) + off)) : len;
    const T *kp = a.k.at(at.b, hk), *vp = a.v.at(at.b, hk);
    Stage<T, D> ks, vs;
    ks.load(kp, a.k.token, 0, all, a.dim);
    vs.load(vp, a.v.token, 0, all, a.dim);

    F qf[D / 16], df[D / 16];
    float delta = 0.0f;
    {
        const T *qp = a.q.at(at.b, at.h) + q * a.q.token, *dp = a.d_o.at(at.b, at.h) + q * a.d_o.token;
        const T *op = a.o.at(at.b, at.h) + q * a.o.token;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            qf[c] = row_frag(qp, there, c, a.dim);
            df[c] = row_frag(dp, there, c, a.dim);
            const F of = row_frag(op, there, c, a.dim);
#pragma unroll
            for (int j = 0; j < 8; ++j) delta = __fmaf_rn((float)df[c][j], (float)of[j], delta);
        }
        delta += other_half(delta);
    }
    const int64_t stat = ((int64_t)at.b * a.heads + at.h) * a.nq + q;
    if (there && lane < 32) a.delta[stat] = delta;
    const float c2 = a.scale * LOG2E, ref = there ? reference(a.lse[stat]) : -NEVER;
    f32x16 dq[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dq[db] = f32x16{0};

    for (int k0 = 0; k0 < all; k0 += R) {
        ks.store(kt);
        vs.store(vt);
        __syncthreads();
        if (k0 + R < all) {
            ks.load(kp, a.k.token, k0 + R, all, a.dim);
            vs.load(vp, a.v.token, k0 + R, all, a.dim);
        }
        if (k0 < most) {
            const bool edge = k0 + R > least;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                f32x16 s{0}, dp{0};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    mma(s, load_r<T, D>(kt, 32 * kb, c), qf[c]);
                    mma(dp, load_r<T, D>(vt, 32 * kb, c), df[c]);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(__fmaf_rn(s[r], c2, -ref));
                    s[r] = p * (dp[r] - delta);
                }
                if (edge) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = k0 + 32 * kb + row_of(r) < mine ? s[r] : 0.0f;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const F f = frag_of<T>(s, c);
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) mma(dq[db], load_t<T, D>(kt, 2 * kb + c, 32 * db), f);
                }
            }
        }
        __syncthreads();
    }
    if (there) store_row<T, D>(a.dq.at(at.b, at.h) + q * a.dq.token, dq, a.scale, a.dim);
}

template <typename T, int D>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || D == 64 ? 2 : 1) void kt_attention_dkv_kernel(Args<T> a, int blocks)
{
    constexpr int R = ROWS<T>, QB = R / 32;
    typedef typename Frag<T>::type F;
    __shared__ __align__(16) char qt[Tile<T, D>::bytes(R)], dt[Tile<T, D>::bytes(R)];
    __shared__ __align__(16) float refs[R], deltas[R];
    const int bh = blockIdx.x % (gridDim.x / blocks), k0 = blockIdx.x / (gridDim.x / blocks) * OWN;
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads, group = a.heads / a.kv_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, off = a.nk - a.nq, len = a.keys(b);
    const int first = k0 + wave * 32, key = first + (lane & 31);
    const bool there = key < len;                   // seen by some query; others get gradient 0 (key < nk)
    F kf[D / 16], vf[D / 16];
    {
        const T *kp = a.k.at(b, hk) + key * a.k.token, *vp = a.v.at(b, hk) + key * a.v.token;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            kf[c] = row_frag(kp, there, c, a.dim);
            vf[c] = row_frag(vp, there, c, a.dim);
        }
    }
    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[db] = dv[db] = f32x16{0};
    const float c2 = a.scale * LOG2E;
    // queries [from, nq) see a key of the workgroup; of this wavefront, those from `mine0` on, all of its keys those from `full` on
    const int from = k0 >= len ? a.nq : a.causal ? max(0, k0 - off) / R * R : 0;
    const int mine0 = first >= len ? a.nq : a.causal ? max(0, first - off) : 0;
    const int full = first + 32 > len ? a.nq : a.causal ? max(0, first + 31 - off) : 0;
    const int mine = a.causal ? key - off : 0;      // first query that sees this lane's key

    Stage<T, D> qs, ds;
    float sref, sdelta;
    const int64_t stats = ((int64_t)b * a.heads + hk * group) * a.nq;
    auto load = [&](int g, int q0) {
        const int h = hk * group + g;
        qs.load(a.q.at(b, h), a.q.token, q0, a.nq, a.dim);
        ds.load(a.d_o.at(b, h), a.d_o.token, q0, a.nq, a.dim);
        if (threadIdx.x < R) {
            const bool ok = q0 + (int)threadIdx.x < a.nq;
            const int64_t i = stats + (int64_t)g * a.nq + q0 + threadIdx.x;
            sref = ok ? reference(a.lse[i]) : -NEVER;
            sdelta = ok ? a.delta[i] : 0.0f;
        }
    };
    int g = 0, q0 = from;
    if (q0 < a.nq) load(g, q0);
    while (q0 < a.nq) {
        qs.store(qt);
        ds.store(dt);
        if (threadIdx.x < R) { refs[threadIdx.x] = sref; deltas[threadIdx.x] = sdelta; }
        __syncthreads();
        int ng = g, nq0 = q0 + R;
        if (nq0 >= a.nq && g + 1 < group) { ng = g + 1; nq0 = from; }
        if (nq0 < a.nq) load(ng, nq0);
        if (q0 + R > mine0) {
            const bool edge = q0 < full;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                f32x16 s{0}, dp{0};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    mma(s, load_r<T, D>(qt, 32 * qb, c), kf[c]);
                    mma(dp, load_r<T, D>(dt, 32 * qb, c), vf[c]);
                }
                f32x16 p;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 ref = *(const f32x4 *)(refs + 32 * qb + row_of(4 * i)), delta = *(const f32x4 *)(deltas + 32 * qb + row_of(4 * i));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = 4 * i + j;
                        p[r] = __builtin_amdgcn_exp2f(__fmaf_rn(s[r], c2, -ref[j]));
                        if (edge) p[r] = there && q0 + 32 * qb + row_of(r) >= mine ? p[r] : 0.0f;
                        s[r] = p[r] * (dp[r] - delta[j]);
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const F pf = frag_of<T>(p, c), sf = frag_of<T>(s, c);
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) {
                        mma(dv[db], load_t<T, D>(dt, 2 * qb + c, 32 * db), pf);
                        mma(dk[db], load_t<T, D>(qt, 2 * qb + c, 32 * db), sf);
                    }
                }
            }
        }
        __syncthreads();
        g = ng;
        q0 = nq0;
    }
    if (key < a.nk) {
        store_row<T, D>(a.dk.at(b, hk) + key * a.dk.token, dk, a.scale, a.dim);
        store_row<T, D>(a.dv.at(b, hk) + key * a.dv.token, dv, 1.0f, a.dim);
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

template <typename T, int D> int fwd(const kt_attention *a, const Args<T> &r, hipStream_t s)
{
    const int blocks = (r.nq + OWN - 1) / OWN;
    kt_attention_fwd_kernel<T, D><<<(unsigned)(a->batch * a->heads * blocks), BLOCK, 0, s>>>(r, blocks);
    return (int)hipGetLastError();
}

template <typename T, int D> int bwd(const kt_attention *a, const Args<T> &r, hipStream_t s)
{
    const int qb = (r.nq + OWN - 1) / OWN, kb = (r.nk + OWN - 1) / OWN;
    if (qb) {
        kt_attention_dq_kernel<T, D><<<(unsigned)(a->batch * a->heads * qb), BLOCK, 0, s>>>(r, qb);
        const int e = (int)hipGetLastError();
        if (e) return e;
    }
    if (!kb) return 0;
    kt_attention_dkv_kernel<T, D><<<(unsigned)(a->batch * a->kv_heads * kb), BLOCK, 0, s>>>(r, kb);
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
    return r.dim <= 64 ? fwd<T, 64>(a, r, s) : fwd<T, 128>(a, r, s);
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
    return r.dim <= 64 ? bwd<T, 64>(a, r, s) : bwd<T, 128>(a, r, s);
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
