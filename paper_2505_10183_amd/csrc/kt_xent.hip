// Softmax cross entropy of a linear layer, loss[t] = log sum_v exp(z[t][v]) - z[t][target_t] with z = x w^T, and its gradients
// dz = dloss (exp(z - lse) - [v = target]),  dx = dz w,  dw = dz^T x.  The logits z are nowhere kept.
//
// All of it is products in tiles.  The forward pass leaves of a tile of z the largest value and the sum of the exponentials for every
// token, which a small kernel joins.  The backward pass goes over pieces of the vocabulary: it makes z of a piece again, leaves dz in the
// workspace in the operands' type, and takes the other two products from there; dx is carried from piece to piece in binary32.
// dz is rounded to bf16 as an operand of bf16 products, as attention's probabilities are, in units of the largest dloss (a mean's 1 / tokens would be the same
// error in all).  A target's element is most of its token's gradients and would carry its rounding into all of them, so what that takes of it (Rests) is added to both
// products: gradients stand 1.65 to 1.75e-3 from the definition in norm, as far as one rounding of the result leaves them, instead of 2.0 to 2.8e-3.
//
// Tokens without a target (or with dloss 0) take no part: the backward pass, and the forward pass where it is long, list the others and copy their rows
// of x one after another, so that the products are made of those alone, and what the rows of the others hold reaches nothing.
#include "kt_mfma.h"

namespace {

// ---- a product ---------------------------------------------------------------------
//
// D[m][n] = sum_k A(m, k) B(n, k), a workgroup for a tile of BM x BN.  An operand is `along` k (k adjacent in memory) or across it (m or n
// adjacent).  Its tiles of STEP k are brought by loads that write LDS themselves, some steps ahead, into slots that take turns.  The barrier
// before a step's last products says that all of it is read (its slot is free again) and that the next one has arrived, so that the fragments of the next step's
// first products are read beside the last products of this one: the matrix cores wait for nothing but the barrier itself.
// A fragment is 16 bytes a lane for both types: lane l holds V of k (V c + ... : chunk c of a step, half h = l / 32, k = V (2 c + h) + j) of its row.  The 32 rows of a fragment of A are taken in an order that
// gives a lane of D 16 neighbouring m: register r of half h is row 16 h + r.
// Measured: 16384 tokens of 50304 x 2048 bf16 forward 2.74 to 2.96 ms, 1.14 to 1.23 PFLOP/s (a library product of these sizes that stores z takes 2.82 to 2.96), matrix cores busy
// 62 % of the cycles at a clock that their load brings down; products of 16384 x 8192 x 2048, dz 495 to 535 us, dx 505 to 545, dw 460 to 510.  f32, 4096 of
// 50304 x 768: 126 TFLOP/s.

// Row of the matrix that row i of a fragment holds.
__device__ __forceinline__ int spread_of(int i) { return (i >> 2 & 1) * 16 + (i >> 3) * 4 + (i & 3); }

// Tile and wavefronts: WM x WN of them, each FM x FN products of 32 x 32.
template <int WM_, int WN_, int FM_, int FN_, int SLOTS_> struct Shape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, SLOTS = SLOTS_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32, BLOCK = WM * WN * 64;
};
typedef Shape<2, 4, 4, 2, 2> Big;       // 256 x 256, 8 wavefronts, 128 KiB of LDS
typedef Shape<2, 2, 2, 2, 2> Mid;       // 128 x 128, 4,  64 KiB
typedef Shape<2, 2, 1, 1, 2> Small;     //  64 x  64, 4,  32 KiB
constexpr int ROW = 128;                                                // bytes of k in a step: a line
template <typename T> constexpr int STEP = ROW / (int)sizeof(T);       // k of a step

template <typename T> struct Operand {
    const T *p;
    int64_t ld;
    int count;                      // of m or n; a multiple of 16 bytes where those are adjacent
};

// A binary32 number as three bf16 that add up to it: 8 bits of its significand each, nearest first.  A product of two such numbers is six products of bf16 pairs,
// exact and summed in binary32, and what is left out (of the 2nd and the 3rd part, and of the 3rd ones) is below 2^-24 of it, half a step of binary32: for the
// matrix cores six bf16 products cost six sixteenths of an f32 one.  The log-sum-exp of 1024 tokens of 5003 logits of 4096
// products each is off by 4.4e-7, half a step of its own, where a library product's logits in 32 bits are off by 1.2e-6.  Of a number below 2^-110 bits under 2^-133 are lost.  An infinite one times
// a part that is 0 is NaN, and products of large ones overflow part by part, to infinities of both signs: logits that are not finite are made again from the numbers
// themselves.  (Not so the gradients' products: dz is finite there, and times an infinite weight nothing is.)  Rows of such numbers are groups of 32, a group the 64 bytes of each part one after another.
struct Three {
    uint16_t part[3];
};
constexpr int PLANES = 3, GROUP = 32;
static_assert(sizeof(Three) * GROUP == 64 * PLANES, "pointers to Three count elements, a group at a time");

// A number that is not finite is its first part, and one that would round to infinity is cut off instead.
__device__ __forceinline__ void in_parts(float f, bf16 *part)
{
    const uint32_t bits = as_u(f);
    const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
    float first = (float)(bf16)f;
    if (finite && (as_u(first) & 0x7f800000u) == 0x7f800000u) first = as_f(bits & 0xffff0000u);
    const float left = finite ? f - first : 0.0f, second = (float)(bf16)left;
    part[0] = (bf16)first;
    part[1] = (bf16)second;
    part[2] = (bf16)(left - second);
}
// 8 numbers of a group, from column c % 32 = 0, 8, 16 or 24 on; one.
__device__ __forceinline__ void put_three(Three *group, int c, const float *f)
{
    bf16x8 part[PLANES];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        bf16 of[PLANES];
        in_parts(f[j], of);
#pragma unroll
        for (int p = 0; p < PLANES; ++p) part[p][j] = of[p];
    }
#pragma unroll
    for (int p = 0; p < PLANES; ++p) *(u32x4 *)((char *)group + p * 64 + c * 2) = __builtin_bit_cast(u32x4, part[p]);
}
__device__ __forceinline__ void put_one(Three *group, int c, float f)
{
    bf16 of[PLANES];
    in_parts(f, of);
#pragma unroll
    for (int p = 0; p < PLANES; ++p) *(bf16 *)((char *)group + p * 64 + c * 2) = of[p];
}
__device__ __forceinline__ float get_one(const Three *group, int c)
{
    float f = 0;
#pragma unroll
    for (int p = PLANES - 1; p >= 0; --p) f += (float)*(const bf16 *)((const char *)group + p * 64 + c * 2);
    return f;
}

// A number that a kernel before has written, the same for all.
__device__ __forceinline__ int scalar(const int *p) { return *(const int __attribute__((address_space(4))) *)(uintptr_t)p; }

// Tiles of one operand on their way from memory to LDS, SIDE of m or n by STEP of k.
template <typename T, int SIDE, int BLOCK, bool ALONG, bool SPREAD> struct Bring {
    static constexpr int V = VE<T>, K = STEP<T>, W = ALONG ? K : SIDE, R = ALONG ? SIDE : K, N = R * W / V / BLOCK;
    static_assert(N >= 1, "a chunk for every lane");
    typedef Tile<T, W> Rows;
    const T *p;
    int64_t ld;
    int count, at[N];
    __device__ __forceinline__ static int row_of(int u) { return (threadIdx.x + u * BLOCK) / (W / V); }
    __device__ __forceinline__ static int col_of(int u)
    {
        const int n = threadIdx.x + u * BLOCK;
        return (n % (W / V) ^ Rows::swizzle(n / (W / V))) * V;
    }
    __device__ __forceinline__ Bring(const Operand<T> &o, int first) : p(ALONG ? o.p + first * o.ld : o.p + first), ld(o.ld), count(min(SIDE, o.count - first))
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int r = row_of(u), row = ALONG && SPREAD ? (r & ~31) + spread_of(r & 31) : r, c = col_of(u);
            at[u] = (ALONG ? row : c) < count ? (row * (int)ld + c) * (int)sizeof(T) : INT32_MIN;
        }
    }
    // The steps from k on, `left` of them until the end, into `tile`, as N loads one by one.  What lies past an end is zeros and is not read.
    u32x4 rs;
    uint32_t to;
    __device__ __forceinline__ void aim(char *tile, int k, int left)
    {
        const int up = (min(left, K) + V - 1) / V * V;
        if (ALONG && left < K) {
#pragma unroll
            for (int u = 0; u < N; ++u)
                if (col_of(u) >= up) at[u] = INT32_MIN;
        }
        const uint64_t base = (uint64_t)(ALONG ? p + k : p + k * ld);
        const int bytes = (ALONG ? (count - 1) * (int)ld + up : (min(left, K) - 1) * (int)ld + count) * (int)sizeof(T);
        rs = u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, (uint32_t)bytes, 0x00020000u};
        to = (uint32_t)(uintptr_t)(KT_LDS char *)tile + wave_id() * 1024;
    }
    __device__ __forceinline__ void load(int u) const
    {
        // as Feed::bring
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(to + u * BLOCK * 16), "v"(at[u]), "s"(rs) : "memory");
    }
};

template <typename T> struct Part;
template <> struct Part<bf16> { typedef bf16x8 type; };
template <> struct Part<float> { typedef f32x4 type; };
// Part j of PARTS of a product of two fragments: f32 takes four instructions, each with one k of both halves.  Those that follow each other should
// add to different sums: the next one to the same waits until this one is through.
template <typename T> constexpr int PARTS = sizeof(T) == 2 ? 1 : 4;
template <int J> __device__ __forceinline__ void multiply(f32x16 &d, bf16x8 a, bf16x8 b) { mma(d, a, b); }
template <int J> __device__ __forceinline__ void multiply(f32x16 &d, f32x4 a, f32x4 b) { d = __builtin_amdgcn_mfma_f32_32x32x2f32(a[J], b[J], d, 0, 0, 0); }

// Fragment of 32 m or n from `first` on, chunk c of the step.
template <typename T, int SIDE, bool ALONG, bool SPREAD>
__device__ __forceinline__ typename Part<T>::type fragment(const char *tile, int first, int c)
{
    const int l = threadIdx.x & 63, h = l >> 5;
    if constexpr (ALONG) {
        return *(const typename Part<T>::type *)(tile + Tile<T, STEP<T>>::at(first + (l & 31), 2 * c + h));
    } else if constexpr (sizeof(T) == 2) {
        const int g = l >> 4 & 1, i = l & 15, j = i & 3;
        const int col = first + (SPREAD ? g * 8 + (j & 1) * 16 + (j >> 1) * 4 : g * 16 + j * 4);
        s16x4 v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int row = 16 * c + 8 * h + 4 * k + (i >> 2);
            const char *p = tile + Tile<T, SIDE>::at(row, col >> 3) + (col & 7) * 2;
            v[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KT_LDS s16x4 *)p);
        }
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        const int col = first + (SPREAD ? spread_of(l & 31) : l & 31);
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *(const float *)(tile + Tile<T, SIDE>::at(8 * c + 4 * h + j, col >> 2) + (col & 3) * 4);
        return v;
    }
}

// Tile number `b` of mt x nt: those of one XCD (every eighth workgroup) follow each other, in blocks of ACROSS n by as many m as
// are at work, so that its L2 keeps their operands.
struct Place {
    int m, n;
};
constexpr int ACROSS = 4;
__device__ __forceinline__ Place place(int b, int mt, int nt)
{
    const int all = mt * nt, q = all / 8, r = all % 8, x = b % 8, i = x * q + min(x, r) + b / 8;
    const int group = i / (ACROSS * mt), wide = min(ACROSS, nt - group * ACROSS), j = i - group * ACROSS * mt;
    return Place{j / wide, group * ACROSS + j % wide};
}

// Until all but LATER of this wavefront's loads into LDS have arrived and it has read what it asked LDS for, and until all wavefronts are here.
template <int LATER> __device__ __forceinline__ void meet()
{
    static_assert(LATER < 16, "the low four bits of vmcnt");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LATER) : "memory");
}

// 16 bytes a lane from memory to LDS, the lanes' one after another from `lds` on, which is the same in all of a wavefront's.
__device__ __forceinline__ void to_lds([[maybe_unused]] const void *p, [[maybe_unused]] char *lds)
{
#ifdef __HIP_DEVICE_COMPILE__           // the host pass does not know the builtin
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p, (KT_LDS void *)lds, 16, 0, 0);
#endif
}

// f32 sums are made in sets of as many steps (128 of k), then added to the total: one after another, thousands of products are rounded at the size of all of
// them.  Loss of 200 tokens of 300 x 8192 off by 6.8e-6 and 6.4e-7 (184 and 197 us; a library product in 32 bits 2.1e-6), of 87 of 1153 x 936 2.1e-6 and 3.9e-7 (27.0 and
// 28.6), gradients of 112 of 50304 x 4096 1.4e-6 and 4.0e-7 (1415 and 1437); in three parts the loss of 8192 of 50304 x 768 7.0e-7 and 1.6e-7 (2984 and 3048).
// With sets of 256 of k the loss of 87 of 1153 x 936 is off by 6.2e-7 (28.2).  bf16 operands bring their own 2^-9, and 16 of them are summed by one instruction: no sets.
constexpr int SET = 4;
template <int FM, int FN> __device__ __forceinline__ void collect(f32x16 (&total)[FM][FN], f32x16 (&acc)[FM][FN])
{
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            total[m][n] += acc[m][n];
            acc[m][n] = f32x16{0};
        }
}

// bf16: what rounding takes from a target's element of dz (in its units), which is most of a token's gradients: 2^-9 of them where nothing makes up for it.  dx adds
// it times the target's row of the weight to its sums; for the weight's gradient a tile adds it times the rows of x whose target is one of its own.  Without and with it, us:
// 16384 tokens of 50304 x 2048 9230 and 9360, 4099 of 5003 x 1001 (then the table's gradient) 201 and 211, 810 of 1000 x 1024 38.0 and 44.1, 15329 of 300 x 1024, whose tiles
// have nearly all tokens each, 91.6 and 114, one of 50304 x 2048 148 and 155.
struct Rests {
    const float *rest;              // of each row of the list, or null: none
    const int *goals;               // its target
    int first;                      // dw: of the piece of the vocabulary
    const void *w;                  // dx: the weight, rows ldw apart
    int64_t ldw;
};

// live: how many of n (B along k) or of the steps (B across) there are, or null: all.
// E: what becomes of the tile.  E::skip(n0, count): nothing to multiply;  E::begin(acc, ...) the sums' start;  E::end(acc, ...).
// f32: no more registers than two workgroups to a CU have, which sets without the bound pass (gradients of 112 of 50304 x 4096 1728 us instead of 1437).
template <typename T, typename S, bool AA, bool BA, typename E>
__global__ __launch_bounds__(S::BLOCK, sizeof(T) == 4 ? 2 : 1) void kt_xent_product_kernel(Operand<T> a, Operand<T> b, int steps, int piece, const int *live, int mt, int nt, E e)
{
    constexpr int K = STEP<T>;
    typedef Bring<T, S::BM, S::BLOCK, AA, true> BringA;
    typedef Bring<T, S::BN, S::BLOCK, BA, false> BringB;
    typedef typename Part<T>::type F;
    constexpr int ABYTES = S::BM * ROW, SLOT = (S::BM + S::BN) * ROW, LOADS = BringA::N + BringB::N, SLOTS = S::SLOTS;
    extern __shared__ __align__(16) char lds[];             // SLOTS slots

    const int wave = wave_id(), lane = threadIdx.x & 63;
    if (live) {
        const int n = scalar(live);
        if constexpr (BA) {
            nt = (n + S::BN - 1) / S::BN;
            if ((int)blockIdx.x >= mt * nt) return;
        } else {
            steps = n;
            piece = ((n + (int)gridDim.y - 1) / (int)gridDim.y + 63) / 64 * 64;
        }
    }
    const Place at = place(blockIdx.x, mt, nt);
    const int m0 = at.m * S::BM, n0 = at.n * S::BN, wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
    const int k0 = blockIdx.y * piece, k1 = min(steps, k0 + piece);
    const int64_t holder = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (S::WM * S::WN) + wave;

    constexpr bool SETS = sizeof(T) == 4;
    f32x16 acc[S::FM][S::FN], total[S::FM][S::FN];         // (without sets: acc alone)
#pragma unroll
    for (int m = 0; m < S::FM; ++m)
#pragma unroll
        for (int n = 0; n < S::FN; ++n) acc[m][n] = total[m][n] = f32x16{0};
    if (!e.skip(n0, S::BN)) {
        BringA from_a(a, m0);
        BringB from_b(b, n0);
        auto aim = [&](char *to, int k) __attribute__((always_inline)) {
            from_a.aim(to, k, k1 - k);
            from_b.aim(to + ABYTES, k, k1 - k);
        };
        auto load = [&](auto u0) __attribute__((always_inline)) {
            constexpr int u = u0;
            if constexpr (u < BringA::N) from_a.load(u);
            else from_b.load(u - BringA::N);
        };
        constexpr int PER = S::FM * S::FN, ALL = PER * PARTS<T>, CHUNKS = ROW / 32, READS = S::FM + S::FN;
        static_assert(CHUNKS % 2 == 0, "two sets of fragments take turns");
        F fa[2][S::FM], fb[2][S::FN];
        // fragment number r of a chunk, in the order in which the products need them
        auto read = [&](const char *slot, auto c0, auto r0) __attribute__((always_inline)) {
            constexpr int c = c0, r = r0;
            if constexpr (r == 0) fa[c % 2][0] = fragment<T, S::BM, AA, true>(slot, wm, c);
            else if constexpr (r <= S::FN) fb[c % 2][r - 1] = fragment<T, S::BN, BA, false>(slot + ABYTES, wn + 32 * (r - 1), c);
            else fa[c % 2][r - S::FN] = fragment<T, S::BM, AA, true>(slot, wm + 32 * (r - S::FN), c);
        };
        int k = k0, ahead = 0;            // the next step to bring; steps brought and not done
        for (; ahead < SLOTS && k < k1; ++ahead, k += K) {
            aim(lds + ahead * SLOT, k);
            span<0, LOADS>(load);
        }
        if constexpr (SETS) e.begin(total, holder);
        else e.begin(acc, holder);
        meet<0>();
        span<0, READS>([&](auto r) { read(lds, std::integral_constant<int, 0>(), r); });
        __builtin_amdgcn_sched_barrier(0);
        int slot = 0;
        auto step = [&]() __attribute__((always_inline)) {
            const int after = slot + 1 == SLOTS ? 0 : slot + 1;
            char *const now = lds + slot * SLOT, *const then = lds + after * SLOT;
            const bool more = k < k1;
            span<0, CHUNKS * ALL>([&](auto n1) {
                constexpr int n = n1 % ALL, c = n1 / ALL, i = n % PER;
                if constexpr (c == CHUNKS - 1 && n == 0) {
                    if (ahead == SLOTS) meet<(SLOTS - 2) * LOADS>();
                    else meet<0>();
                    if (more) {
                        aim(now, k);
                        // bf16: all loads at once (spread over the products that follow the decoder's backward pass takes 9.87 ms instead of 9.47); f32, whose
                        // products take eight times as long: spread (4096 x 50304 x 768 7.55 ms instead of 8.10)
                        if constexpr (PARTS<T> == 1) span<0, LOADS>(load);
                    }
                }
                multiply<n / PER>(acc[i / S::FN][i % S::FN], fa[c % 2][i / S::FN], fb[c % 2][i % S::FN]);
                // beside each product from the first on, so that the last ones are there for the next chunk's first products
                constexpr int RATE = (READS + ALL - 1) / ALL;
                span<(n * RATE < READS ? n * RATE : READS), ((n + 1) * RATE < READS ? (n + 1) * RATE : READS)>([&](auto r) {
                    read(c + 1 < CHUNKS ? now : then, std::integral_constant<int, (c + 1) % CHUNKS>(), r);
                });
                if constexpr (c == CHUNKS - 1 && PARTS<T> > 1) {
                    if (more) span<n * LOADS / ALL, (n + 1) * LOADS / ALL>(load);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            if (more) k += K;
            else --ahead;
            slot = after;
        };
        if constexpr (SETS) {
            while (ahead > 0) {
#pragma unroll 1
                for (int n = 0; n < SET && ahead > 0; ++n) step();
                collect(total, acc);
            }
        } else {
            while (ahead > 0) step();
        }
    }
    if constexpr (SETS) collect(acc, total);                // acc is 0
    if constexpr (E::TARGETS) {
        // Rests: products of the rows of x whose target is one of this tile's n with a matrix of their rests and zeros.  The rows, of the tokens that this workgroup has gone
        // through, are listed up to LIST of them at a time in the other slot; 64 of them are a step.
        static_assert(!AA && !BA && sizeof(T) == 2, "the weight's gradient in bf16");
        constexpr int LIST = 4096, WAVES = S::BLOCK / 64, EACH = LIST / S::BLOCK, MOST = 64;
        static_assert(SLOTS >= 2 && LIST * 4 <= SLOT && K == MOST, "a slot holds the list");
        struct Own {
            int n;
            float rest;
        };
        Own *const own = (Own *)(lds + ABYTES);
        int *const counts = (int *)(own + MOST), *const list = (int *)(lds + SLOT);
        const int there = min(S::BM, a.count - m0);
        for (int base = k0; base < k1; base += LIST) {
            int goal[EACH], n = 0;
            const int mine = base + wave * (LIST / WAVES) + lane;
#pragma unroll
            for (int u = 0; u < EACH; ++u) goal[u] = mine + u * 64 < k1 ? e.rests.goals[mine + u * 64] - e.rests.first - n0 : -1;
#pragma unroll
            for (int u = 0; u < EACH; ++u) n += __popcll(__ballot(goal[u] >= 0 && goal[u] < S::BN));
            meet<0>();                                      // LDS is read
            if (lane == 0) counts[wave] = n;
            meet<0>();
            int before = 0, all = 0;
            for (int w = 0; w < WAVES; ++w) {
                before += w < wave ? counts[w] : 0;
                all += counts[w];
            }
            all = __builtin_amdgcn_readfirstlane(all);
            if (all == 0) continue;
#pragma unroll
            for (int u = 0; u < EACH; ++u) {
                const bool here = goal[u] >= 0 && goal[u] < S::BN;
                const uint64_t word = __ballot(here);
                if (here) list[before + __popcll(word & ((1ull << lane) - 1))] = mine + u * 64;
                before += __popcll(word);
            }
            meet<0>();
            for (int s = 0; s < all; s += MOST) {
                const int left = all - s;
#pragma unroll
                for (int u = 0; u < BringA::N; ++u) {
                    // rows past the list's end meet zeros only, and columns past the width are nobody's: any of them will do
                    const int row = list[s + min(BringA::row_of(u), left - 1)], c = BringA::col_of(u);
                    to_lds(a.p + row * a.ld + m0 + (c < there ? c : 0), lds + wave * 1024 + u * (S::BLOCK * 16));
                }
                if (wave == 0) {
                    Own o{-1, 0.0f};
                    if (lane < left) {
                        const int row = list[s + lane];
                        o = Own{e.rests.goals[row] - e.rests.first - n0, e.rests.rest[row]};
                    }
                    own[lane] = o;
                }
                meet<0>();
#pragma unroll
                for (int c = 0; c < ROW / 32; ++c) {
                    if (16 * c >= left) break;
                    F fa[S::FM], fb[S::FN];
#pragma unroll
                    for (int i = 0; i < S::FM; ++i) fa[i] = fragment<T, S::BM, AA, true>(lds, wm + 32 * i, c);
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const Own o = own[16 * c + 8 * (lane >> 5) + q];
#pragma unroll
                        for (int j = 0; j < S::FN; ++j) fb[j][q] = o.n == wn + 32 * j + (lane & 31) ? (T)o.rest : (T)0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < S::FM; ++i)
#pragma unroll
                        for (int j = 0; j < S::FN; ++j) multiply<0>(acc[i][j], fa[i], fb[j]);
                }
                meet<0>();
            }
        }
    }
    if constexpr (E::ROWS) __syncthreads();                 // LDS is read: the epilogue takes it
    e.end(acc, m0 + wm + (lane >> 5) * 16, n0 + wn + (lane & 31), holder, wave / S::WN + S::WM * at.m, lds + wave * (S::FM * 4096));
}

// The same product of numbers in three parts: tiles of 256 x 128, 32 of k a step, each part a tile of its own in LDS (144 KiB of two slots).  Six products
// share each fragment, so LDS is busy 13 to 17 % of the cycles and the matrix cores 50 to 64 %: 8192 x 50304 x 768 at 210 TFLOP/s of f32 products, 1.26 PFLOP/s of
// bf16 ones, where f32 instructions reach 131.
template <int SIDE, int BLOCK, bool ALONG, bool SPREAD> struct BringThree {
    static constexpr int K = GROUP, PART = SIDE * K / 8, N = PLANES * PART / BLOCK;       // 16-byte chunks of a part; a lane's
    static_assert(PLANES * PART % BLOCK == 0, "a chunk for every lane");
    typedef Tile<bf16, SIDE> Across;
    const Three *p;
    int64_t ld;
    int count, at[N];
    u32x4 rs;
    uint32_t to;
    // rows of 64 bytes, four of which fill the banks: 16 lanes that read the same chunk of 16 rows read all of them
    __device__ __forceinline__ static int along(int row, int chunk) { return row * 64 + (chunk ^ (row >> 2 & 3)) * 16; }
    __device__ __forceinline__ BringThree(const Operand<Three> &o, int first) : p(ALONG ? o.p + first * o.ld : o.p + first), ld(o.ld), count(min(SIDE, o.count - first))
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int n = threadIdx.x + u * BLOCK, part = n / PART, m = n % PART;
            if (ALONG) {
                const int r = m / 4, row = SPREAD ? (r & ~31) + spread_of(r & 31) : r;
                at[u] = row < count ? row * (int)ld * (int)sizeof(Three) + part * 64 + (m % 4 ^ (r >> 2 & 3)) * 16 : INT32_MIN;
            } else {
                const int r = m / (SIDE / 8), c = (m % (SIDE / 8) ^ Across::swizzle(r)) * 8;
                at[u] = c < count ? (r * (int)ld + c / GROUP * GROUP) * (int)sizeof(Three) + part * 64 + c % GROUP * 2 : INT32_MIN;
            }
        }
    }
    __device__ __forceinline__ void aim(char *tile, int k, int left)
    {
        const uint64_t base = (uint64_t)(ALONG ? p + k : p + k * ld);
        const int bytes = (ALONG ? (count - 1) * (int)ld + K : (min(left, K) - 1) * (int)ld + count) * (int)sizeof(Three);
        rs = u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, (uint32_t)bytes, 0x00020000u};
        to = (uint32_t)(uintptr_t)(KT_LDS char *)tile + wave_id() * 1024;
    }
    __device__ __forceinline__ void load(int u) const
    {
        // as Feed::bring
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(to + u * BLOCK * 16), "v"(at[u]), "s"(rs) : "memory");
    }
    // 32 m or n from `first` on, 16 of k from 16 c on
    static __device__ __forceinline__ bf16x8 read(const char *tile, int part, int first, int c)
    {
        const char *const t = tile + part * SIDE * 64;
        if constexpr (ALONG) return *(const bf16x8 *)(t + along(first + (threadIdx.x & 31), 2 * c + (threadIdx.x >> 5 & 1)));
        else return fragment<bf16, SIDE, false, SPREAD>(t, first, c);
    }
    // the same of the numbers themselves
    static __device__ __forceinline__ f32x8 numbers(const char *tile, int first, int c)
    {
        f32x8 v = __builtin_convertvector(read(tile, PLANES - 1, first, c), f32x8);
#pragma unroll
        for (int p = PLANES - 2; p >= 0; --p) v += __builtin_convertvector(read(tile, p, first, c), f32x8);
        return v;
    }
};

struct Split {
    static constexpr int WM = 4, WN = 2, FM = 2, FN = 2, BM = WM * FM * 32, BN = WN * FN * 32, BLOCK = WM * WN * 64, SLOT = (BM + BN) * 64 * PLANES;
};
template <bool AA, bool BA, typename E>
__global__ __launch_bounds__(Split::BLOCK) void kt_xent_three_kernel(Operand<Three> a, Operand<Three> b, int steps, int piece, const int *live, int mt, int nt, E e)
{
    typedef Split S;
    typedef BringThree<S::BM, S::BLOCK, AA, true> BringA;
    typedef BringThree<S::BN, S::BLOCK, BA, false> BringB;
    constexpr int K = GROUP, ABYTES = S::BM * 64 * PLANES, LA = BringA::N, LB = BringB::N;
    extern __shared__ __align__(16) char lds[];             // two slots

    const int wave = wave_id(), lane = threadIdx.x & 63;
    if (live) {
        const int n = scalar(live);
        if constexpr (BA) {
            nt = (n + S::BN - 1) / S::BN;
            if ((int)blockIdx.x >= mt * nt) return;
        } else {
            steps = n;
            piece = ((n + (int)gridDim.y - 1) / (int)gridDim.y + 63) / 64 * 64;
        }
    }
    const Place at = place(blockIdx.x, mt, nt);
    const int m0 = at.m * S::BM, n0 = at.n * S::BN, wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
    const int k0 = blockIdx.y * piece, k1 = min(steps, k0 + piece);

    f32x16 acc[S::FM][S::FN], total[S::FM][S::FN];
#pragma unroll
    for (int m = 0; m < S::FM; ++m)
#pragma unroll
        for (int n = 0; n < S::FN; ++n) acc[m][n] = total[m][n] = f32x16{0};
    BringA from_a(a, m0);
    BringB from_b(b, n0);
    auto bring = [&](char *to, int k) __attribute__((always_inline)) {
        from_a.aim(to, k, k1 - k);
        from_b.aim(to + ABYTES, k, k1 - k);
        span<0, LA>([&](auto u) { from_a.load(u); });
        span<0, LB>([&](auto u) { from_b.load(u); });
    };
    // the products of two numbers' parts, least first
    constexpr int PER = S::FM * S::FN, PAIRS = 6, ALL = PER * PAIRS, READS = (S::FM + S::FN) * PLANES;
    constexpr int PA[PAIRS] = {2, 1, 0, 1, 0, 0}, PB[PAIRS] = {0, 1, 2, 0, 1, 0};
    bf16x8 fa[2][PLANES][S::FM], fb[2][PLANES][S::FN];
    // fragment number r of a chunk, in the order in which the products need them: parts 2 of A and 0 of B first
    auto read = [&](const char *slot, auto c0, auto r0) __attribute__((always_inline)) {
        constexpr int c = c0, r = r0, group = r / 2, i = r % 2, part = group / 2;
        static_assert(S::FM == 2 && S::FN == 2, "two fragments of each part");
        if constexpr (group % 2 == 0) fa[c][PLANES - 1 - part][i] = BringA::read(slot, PLANES - 1 - part, wm + 32 * i, c);
        else fb[c][part][i] = BringB::read(slot + ABYTES, part, wn + 32 * i, c);
    };
    int k = k0, ahead = 0;
    for (; ahead < 2 && k < k1; ++ahead, k += K) bring(lds + ahead * S::SLOT, k);
    const int64_t holder = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (S::WM * S::WN) + wave;
    e.begin(total, holder);
    meet<0>();
    span<0, READS>([&](auto r) { read(lds, std::integral_constant<int, 0>(), r); });
    __builtin_amdgcn_sched_barrier(0);
    int slot = 0;
    auto step = [&]() __attribute__((always_inline)) {
        char *const now = lds + slot * S::SLOT, *const then = lds + (slot ^ 1) * S::SLOT;
        const bool more = k < k1;
        span<0, 2 * ALL>([&](auto n1) {
            constexpr int c = n1 / ALL, n = n1 % ALL, pair = n / PER, i = n % PER / S::FN, j = n % S::FN;
            if constexpr (c == 1 && n == 0) {
                meet<0>();
                if (more) bring(now, k);
            }
            mma(acc[i][j], fa[c][PA[pair]][i], fb[c][PB[pair]][j]);
            if constexpr (n < READS) read(c == 0 ? now : then, std::integral_constant<int, 1 - c>(), std::integral_constant<int, n>());
            __builtin_amdgcn_sched_barrier(0);
        });
        if (more) k += K;
        else --ahead;
        slot ^= 1;
    };
    while (ahead > 0) {
#pragma unroll 1
        for (int n = 0; n < SET && ahead > 0; ++n) step();
        collect(total, acc);
    }
    collect(acc, total);
    if constexpr (E::LOGITS) {
        // Sums times 0 are 0 if they are finite; those of rows past the list, which hold anything, do not count.  4096 tokens of 50304 x 768 forward: 1.95 ms with this look
        // and without; with a token of NaN, whose tiles all fall to a few CUs, 5.2, with nothing else 5.0.
        const int rows = live ? scalar(live) : b.count;
        bool not_finite = false;
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            float zero[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) zero[r % 2] = __builtin_fmaf(acc[i][j][r], 0.0f, zero[r % 2]);
            not_finite |= !(zero[0] + zero[1] == 0.0f) && n0 + wn + 32 * j + (lane & 31) < rows;
        }
        const bool mine = __ballot(not_finite) != 0;
        int *const odd = (int *)lds;
        __syncthreads();                                    // LDS is read
        if (lane == 0) odd[wave] = mine;
        __syncthreads();
        int any = 0;
        for (int w = 0; w < S::WM * S::WN; ++w) any |= odd[w];
        if (__builtin_amdgcn_readfirstlane(any)) {
            __syncthreads();                                // all have read what the others say
            f32x16 sum[S::FM][S::FN];
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j) sum[i][j] = f32x16{0};
#pragma unroll 1
            for (k = k0; k < k1; k += K) {
                bring(lds, k);
                meet<0>();
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    f32x8 na[S::FM], nb[S::FN];
#pragma unroll
                    for (int i = 0; i < S::FM; ++i) na[i] = BringA::numbers(lds, wm + 32 * i, c);
#pragma unroll
                    for (int j = 0; j < S::FN; ++j) nb[j] = BringB::numbers(lds + ABYTES, wn + 32 * j, c);
#pragma unroll
                    for (int i = 0; i < S::FM; ++i)
#pragma unroll
                        for (int j = 0; j < S::FN; ++j) mma(sum[i][j], na[i], nb[j]);
                }
                meet<0>();
            }
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = fabsf(acc[i][j][r]) < INFINITY ? acc[i][j][r] : sum[i][j][r];
        }
    }
    if constexpr (E::ROWS) __syncthreads();                 // LDS is read: the epilogue takes it
    e.end(acc, m0 + wm + (lane >> 5) * 16, n0 + wn + (lane & 31), holder, wave / S::WN + S::WM * at.m, lds + wave * (S::FM * 4096));
}

// ---- what becomes of a tile ----------------------------------------------------------

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <typename I> __device__ __forceinline__ int target_of(const I *targets, int n, int tokens, int vocab)
{
    if (n >= tokens) return -1;
    const I t = targets[n];
    return t >= 0 && t < (I)vocab ? (int)t : -1;
}

// 32 rows (lanes) of FM * 32 columns to memory in whole lines: each lane's 16 neighbouring columns go into this wavefront's part of LDS and
// come back a row after the other.  The chunks of a row are exchanged, so that lanes of different rows use different banks.
// f(i, values): the 16 values of column 32 i + 16 h on;  out: the matrix at its first row and this first column;  first, rows, cols: the first row, and what
// of them is there;  map: where a row goes, or null.
template <int FM, typename G, typename F> __device__ __forceinline__ void store_rows(char *scratch, G *out, int64_t ld, int first, int rows, int cols, const int *map, F f)
{
    constexpr int CHUNKS = FM * 32 / VE<G>;
    static_assert((CHUNKS & (CHUNKS - 1)) == 0, "chunks of a row are exchanged among a power of two");
    const int lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
    u32x4 *const to = (u32x4 *)scratch;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        float v[16];
        f(i, v);
#pragma unroll
        for (int c = 0; c < 16; c += VE<G>) to[l * CHUNKS + (((32 * i + 16 * h + c) / VE<G>) ^ (l & (CHUNKS - 1)))] = narrow<G>(v + c);
    }
    __builtin_amdgcn_wave_barrier();                        // of one wavefront: LDS serves it in order
#pragma unroll
    for (int u = 0; u < 32 * CHUNKS / 64; ++u) {
        const int n = u * 64 + lane, row = n / CHUNKS, c = n % CHUNKS;
        const u32x4 v = to[row * CHUNKS + (c ^ (row & (CHUNKS - 1)))];
        if (row < rows && c * VE<G> < cols) st_chunk(out + (map ? map[first + row] : first + row) * ld, c * VE<G>, cols, v);
    }
}

// Forward: for a wavefront's vocabulary rows the largest logit of each token and the sum of the exponentials over it; the
// target's logit.
template <typename I> struct Stats {
    static constexpr bool ROWS = false, LOGITS = true, TARGETS = false;
    f32x2 *parts;                   // [part][tokens]
    float *hit;                     // [tokens]
    const I *targets;
    const int *map, *live;          // the token of each row of x and their number, or null: all tokens
    int tokens, vocab, first, end_;         // the piece of the vocabulary: rows [first, end)
    int part0;
    __device__ __forceinline__ bool skip(int n0, int count) const
    {
        if (live) return false;
        bool any = false;       // every wavefront for itself
        for (int i = threadIdx.x & 63; i < count; i += 64) any |= target_of(targets, n0 + i, tokens, vocab) >= 0;
        return __ballot(any) == 0;
    }
    template <typename A> __device__ __forceinline__ void begin(A &, int64_t) const {}
    template <int FM, int FN> __device__ __forceinline__ void end(f32x16 (&acc)[FM][FN], int m, int n, int64_t, int part, char *) const
    {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            int t = n + 32 * j;
            if (live) t = t < scalar(live) ? map[t] : tokens;
            const int want = target_of(targets, t, tokens, vocab) - first - m, room = end_ - first - m;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if (room < 32 * i + 16) {                   // past the vocabulary
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = 32 * i + r >= room ? -INFINITY : acc[i][j][r];
                }
                if ((uint32_t)(want - 32 * i) < 16) {
                    float at = 0;
#pragma unroll
                    for (int r = 0; r < 16; ++r) at = 32 * i + r == want ? acc[i][j][r] : at;
                    hit[t] = at;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * LOG2E);
            sum += __shfl_xor(sum, 32);
            if ((threadIdx.x & 32) == 0 && t < tokens) parts[(int64_t)(part0 + part) * tokens + t] = f32x2{top, sum};
        }
    }
    __device__ __forceinline__ void few(f32x4 z, int v, int t, int part) const
    {
        const int want = target_of(targets, t, tokens, vocab) - first - v, room = end_ - first - v;
        float top = -INFINITY, sum = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (r == want) hit[t] = z[r];
            z[r] = r < room ? z[r] : -INFINITY;
            top = fmaxf(top, z[r]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((z[r] - base) * LOG2E);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (threadIdx.x % 64 < 16 && t < tokens) parts[(int64_t)(part0 + part) * tokens + t] = f32x2{top, sum};
    }
};

// Backward: dz of a piece of the vocabulary, rows of tokens `ld` apart; columns past the vocabulary are zeros.
template <typename T, typename I> struct Slope {
    static constexpr bool ROWS = true, LOGITS = true, TARGETS = false, HALVES = std::is_same_v<T, bf16>;
    T *dz;
    int64_t ld;
    const float *lse, *dloss, *unit;
    float *others;                  // [row][part of `parts`]: what the exponentials of other rows than the target's add up to, or null
    const I *targets;
    const int *map, *live;          // the token of each row, and their number
    int tokens, vocab, first, end_, parts;
    float *rest;                    // [row], bf16: what rounding takes from the target's element
    __device__ __forceinline__ bool skip(int, int) const { return false; }
    template <typename A> __device__ __forceinline__ void begin(A &, int64_t) const {}
    __device__ __forceinline__ float share(int at) const { return HALVES ? dloss[at] / *unit : dloss[at]; }
    template <int FM, int FN> __device__ __forceinline__ void end(f32x16 (&acc)[FM][FN], int m, int n, int64_t, int part, char *scratch) const
    {
        const int h = threadIdx.x >> 5 & 1, l = threadIdx.x & 31, m0 = m - 16 * h;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int row = n + 32 * j, first_row = row - l, rows = scalar(live);
            if (first_row >= rows) continue;
            const int at = map[min(row, rows - 1)], target = (int)targets[at] - first, room = end_ - first;
            const float up = share(at), base = lse[at];
            float sum = 0, hit = 0;
            auto values = [&](int i, float *f) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int v = m + 32 * i + r;
                    const float e = __builtin_amdgcn_exp2f((acc[i][j][r] - base) * LOG2E), p = e - (v == target ? 1.0f : 0.0f);
                    f[r] = v < room ? p * up : 0.0f;
                    if constexpr (!HALVES) sum += v < room && v != target ? e : 0.0f;
                    else hit = v == target ? f[r] : hit;
                }
            };
            if constexpr (std::is_same_v<T, Three>) {
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    float f[16];
                    values(i, f);
                    if (row >= rows || m0 + 32 * i >= ld) continue;
                    Three *group = dz + row * ld + m0 + 32 * i;
                    put_three(group, 16 * h, f);
                    put_three(group, 16 * h + 8, f + 8);
                }
            } else {
                store_rows<FM>(scratch, dz + m0, ld, first_row, rows - first_row, (int)ld - m0, nullptr, values);
            }
            if constexpr (!HALVES) {
                sum += __shfl_xor(sum, 32);
                if (others && h == 0 && row < rows) others[(int64_t)row * parts + part] = sum;
            } else {
                // 16 of each 32 columns are this lane's
                const int in = target - m;
                if (in >= 0 && in < FM * 32 && in % 32 < 16 && row < rows) rest[row] = hit - (float)(bf16)hit;
            }
        }
    }
    __device__ __forceinline__ void few(f32x4 z, int v, int t, int part) const
    {
        if (t >= scalar(live)) return;
        const int at = map[t], want = (int)targets[at] - first - v, room = end_ - first - v;
        const float up = share(at), base = lse[at];
        T f[4];
        float sum = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float e = __builtin_amdgcn_exp2f((z[r] - base) * LOG2E), p = e - (r == want ? 1.0f : 0.0f);
            f[r] = (T)(r < room ? p * up : 0.0f);
            sum += r < room && r != want ? e : 0.0f;
            if constexpr (HALVES) {
                if (r == want) rest[t] = p * up - (float)f[r];
            }
        }
        if constexpr (!HALVES) {
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (others && (threadIdx.x & 63) < 16) others[(int64_t)t * parts + part] = sum;
        }
        if (v >= ld) return;
        T *row = dz + t * ld + v;
        if constexpr (HALVES) *(u32x2 *)row = __builtin_bit_cast(u32x2, f);
        else *(u32x4 *)row = __builtin_bit_cast(u32x4, f);
    }
};

// f32: exp(z - lse) - 1 of a target that is likely is a difference of near numbers, off by what z and lse are, and is
// taken from the others' exponentials, which add up to what it lacks of 1.  (Below 1/2 the difference is the nearer one.)  With logits of 4096 products and an
// lse whose roundings are not this layer's the gradients of 4 tokens of 1000 were off by 2.1e-5 of their norm.  A wavefront a token: 3 us at a few.
template <typename X, typename I>
__global__ __launch_bounds__(256) void kt_xent_target_kernel(X *dz, int64_t ld, const float *others, int parts, const float *dloss, const I *targets, const int *map,
                                                             const int *live)
{
    const int row = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (row >= *live) return;
    const float *of = others + (int64_t)row * parts;
    float sum = 0;
#pragma unroll 8
    for (int k = lane; k < parts; k += 64) sum += of[k];
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (lane || !(sum < 0.5f)) return;
    const int at = map[row], v = (int)targets[at];
    const float f = -sum * dloss[at];
    if constexpr (std::is_same_v<X, Three>) put_one(dz + row * ld + v / GROUP * GROUP, v % GROUP, f);
    else dz[row * ld + v] = f;
}

// The same where the vocabulary is several pieces: what the others add up to is known behind the last of them, when the target's piece has long been multiplied.  So
// the element that was taken there is kept, and what the others say instead of it is added to the results.  Rows of the list whose element stands as it was
// are left alone.  130 tokens of 5001 x 8191 with likely targets: elements of the gradients off by 4 % without.  It takes 44 us of 5380 of 4096 tokens of
// 50304 x 768, 28 of 1120 of 70 tokens of 9500 x 8191.
template <typename X, typename I>
__global__ __launch_bounds__(256) void kt_xent_others_kernel(const X *dz, int64_t ld, const float *others, int parts, const I *targets, const int *map, const int *live,
                                                             int first, int end, float *sums, float *taken)
{
    const int row = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (row >= *live) return;
    const float *of = others + (int64_t)row * parts;
    float sum = 0;
#pragma unroll 8
    for (int k = lane; k < parts; k += 64) sum += of[k];
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (lane) return;
    sums[row] = first ? sums[row] + sum : sum;
    const int v = (int)targets[map[row]] - first;
    if (v < 0 || v >= end - first) return;
    if constexpr (std::is_same_v<X, Three>) taken[row] = get_one(dz + row * ld + v / GROUP * GROUP, v % GROUP);
    else taken[row] = dz[row * ld + v];
}
// dx of each row that changes; for dw the rows `to` that its targets' rows get, and ids: the target, or -1 where there is nothing to add.
template <typename I>
__global__ __launch_bounds__(256) void kt_xent_likely_kernel(const float *sums, const float *taken, const float *dloss, const I *targets, const int *map, const int *live,
                                                             int tokens, int width, const float *x, int64_t ldx, const float *w, int64_t ldw, float *dx, int64_t lddx,
                                                             float *to, int64_t ldto, int *ids)
{
    const int parts = (width + 255) / 256, count = *live;
    for (int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; n < (int64_t)tokens * parts; n += (int64_t)gridDim.x * 4) {
        const int row = (int)(n / parts), part = (int)(n % parts), lane = threadIdx.x & 63;
        int at = 0, target = -1;
        float more = 0;
        if (row < count && sums[row] < 0.5f) {
            at = map[row];
            more = -sums[row] * dloss[at] - taken[row];
            if (more != 0.0f) target = (int)targets[at];
        }
        if (ids && part == 0 && lane == 0) ids[row] = target;
        if (target < 0) continue;
        const int c = part * 256 + lane * 4;
        float a[4], b[4];
        if (dx) {
            widen<float>(ld_chunk(w + target * ldw, c, width), a);
            widen<float>(ld_chunk(dx + at * lddx, c, width), b);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] += more * a[j];
            st_chunk(dx + at * lddx, c, width, narrow<float>(b));
        }
        if (ids) {
            widen<float>(ld_chunk(x + at * ldx, c, width), a);
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] *= more;
            st_chunk(to + row * ldto, c, width, narrow<float>(a));
        }
    }
}

// Sums that the next piece of the vocabulary goes on with, as the lanes hold them: nobody else reads them.  `holder`: the wavefront's number.
template <int FM, int FN> __device__ __forceinline__ void resume(const float *sums, int64_t holder, f32x16 (&acc)[FM][FN])
{
    const float *p = sums + holder * (FM * FN * 1024) + (threadIdx.x & 63) * 4;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const u32x4 v = *(const u32x4 *)(p + ((i * FN + j) * 4 + c) * 256);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][4 * c + r] = as_f(v[r]);
            }
}
struct Carry {
    static constexpr bool ROWS = false, LOGITS = false, TARGETS = false;
    float *sums;
    bool first;
    __device__ __forceinline__ bool skip(int, int) const { return false; }
    template <int FM, int FN> __device__ __forceinline__ void begin(f32x16 (&acc)[FM][FN], int64_t holder) const
    {
        if (!first) resume(sums, holder, acc);
    }
    template <int FM, int FN> __device__ __forceinline__ void end(f32x16 (&acc)[FM][FN], int, int, int64_t holder, int, char *) const
    {
        float *p = sums + holder * (FM * FN * 1024) + (threadIdx.x & 63) * 4;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    u32x4 v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = as_u(acc[i][j][4 * c + r]);
                    *(u32x4 *)(p + ((i * FN + j) * 4 + c) * 256) = v;
                }
    }
};

// The result, or (G = float, pieces of k) the sums of a piece.
template <typename G, bool TARGETS_ = false> struct Result {
    static constexpr bool ROWS = true, LOGITS = false, TARGETS = TARGETS_;
    G *out;
    int64_t ld, apart;              // rows; matrices of the pieces of k
    const float *sums;              // what Carry left, or null
    const int *map, *live;          // where a row goes, and how many there are, or null
    const float *unit;              // what the sums are in, or null: 1
    int rows, cols;
    Rests rests;                    // bf16
    __device__ __forceinline__ bool skip(int, int) const { return false; }
    template <int FM, int FN> __device__ __forceinline__ void begin(f32x16 (&acc)[FM][FN], int64_t holder) const
    {
        if (sums) resume(sums, holder, acc);
    }
    template <int FM, int FN> __device__ __forceinline__ void end(f32x16 (&acc)[FM][FN], int m, int n, int64_t, int, char *scratch) const
    {
        const int h = threadIdx.x >> 5 & 1, l = threadIdx.x & 31, m0 = m - 16 * h;
        const float of = unit ? *unit : 1.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int first = n + 32 * j - l, end = live ? scalar(live) : rows;
            if (first >= end || m0 >= cols) continue;
            const G *w = nullptr;
            float more = 0;
            if constexpr (sizeof(G) == 2 && !TARGETS) {
                if (rests.rest && n + 32 * j < end) {
                    more = rests.rest[n + 32 * j];
                    w = static_cast<const G *>(rests.w) + rests.goals[n + 32 * j] * rests.ldw;
                }
            }
            store_rows<FM>(scratch, out + blockIdx.y * apart + m0, ld, first, end - first, cols - m0, map, [&](int i, float *f) {
                if constexpr (sizeof(G) == 2 && !TARGETS) {
                    float g[16];
#pragma unroll
                    for (int r = 0; r < 16; r += 8) widen<G>(w ? ld_chunk(w, m + 32 * i + r, cols) : u32x4{0, 0, 0, 0}, g + r);
#pragma unroll
                    for (int r = 0; r < 16; ++r) f[r] = (acc[i][j][r] + more * g[r]) * of;
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) f[r] = acc[i][j][r] * of;
                }
            });
        }
    }
};

// ---- logits of few tokens --------------------------------------------------------------
//
// Few tokens are bound by the weight's bytes: a wavefront takes 16 rows of it from memory into fragments, 64 bytes of each row a load and AHEAD
// loads on their way, with no LDS and no wait for others.  D = 16 x 16: lane l holds row (A) or token (B) l % 16, k = V (l / 16) + 0.. of 4 V, and of D the
// token l % 16 of rows 4 (l / 16) + 0..3.
constexpr int FEW_AHEAD = 8;

__device__ __forceinline__ void multiply16(f32x4 &d, u32x4 a, u32x4 b, bf16)
{
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), d, 0, 0, 0);
}
__device__ __forceinline__ void multiply16(f32x4 &d, u32x4 a, u32x4 b, float)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) d = __builtin_amdgcn_mfma_f32_16x16x4f32(as_f(a[j]), as_f(b[j]), d, 0, 0, 0);
}

// GROUPS of 16 tokens.  E::few(z, rows from, token, part): four logits of one token.
template <typename T, int GROUPS, typename E>
__global__ __launch_bounds__(64) void kt_xent_few_kernel(const T *w, int64_t ldw, int rows, const T *x, int64_t ldx, int tokens, int width, E e)
{
    constexpr int V = VE<T>, STEP_ = 4 * V;
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4, part = blockIdx.x, v0 = part * 16;
    const T *a = w + min(v0 + l, rows - 1) * ldw + g * V, *b[GROUPS];
    f32x4 z[GROUPS];
#pragma unroll
    for (int t = 0; t < GROUPS; ++t) {
        b[t] = x + min(16 * t + l, tokens - 1) * ldx + g * V;
        z[t] = f32x4{0, 0, 0, 0};
    }
    // two sets of loads take turns: one is on its way while the other is used
    u32x4 ra[2][FEW_AHEAD], rb[2][FEW_AHEAD][GROUPS];
    auto load = [&](auto set0, int k) __attribute__((always_inline)) {
        constexpr int set = set0;
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) {
            ra[set][u] = ld16(a + k + u * STEP_);
#pragma unroll
            for (int t = 0; t < GROUPS; ++t) rb[set][u][t] = ld16(b[t] + k + u * STEP_);
        }
    };
    // a set's sums first, then theirs: 4096 f32 products one after another are off three times as far, at no less time
    auto use = [&](auto set0) __attribute__((always_inline)) {
        constexpr int set = set0;
        f32x4 of[GROUPS];
#pragma unroll
        for (int t = 0; t < GROUPS; ++t) of[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u)
#pragma unroll
            for (int t = 0; t < GROUPS; ++t) multiply16(of[t], ra[set][u], rb[set][u][t], T());
#pragma unroll
        for (int t = 0; t < GROUPS; ++t) z[t] += of[t];
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    constexpr int SET = FEW_AHEAD * STEP_;
    const int whole = width / SET * SET;
    int k = 0;
    if (whole) load(first, 0);
    for (; k < whole; k += 2 * SET) {
        if (k + SET < whole) load(second, k + SET);
        use(first);
        if (k + SET >= whole) break;
        if (k + 2 * SET < whole) load(first, k + 2 * SET);
        use(second);
    }
    k = whole;
    for (; k < width; k += STEP_) {
        const int left = width - k - g * V;
        const u32x4 ra = ld_chunk(a + k, 0, left);
#pragma unroll
        for (int t = 0; t < GROUPS; ++t) multiply16(z[t], ra, ld_chunk(b[t] + k, 0, left), T());
    }
#pragma unroll
    for (int t = 0; t < GROUPS; ++t) e.few(z[t], v0 + 4 * g, 16 * t + l, part);
}

// ---- the small kernels beside them ---------------------------------------------------

// EACH neighbouring elements of a row from column c on as an operand has them; zeros from `cols` on.
template <typename X> constexpr int EACH = std::is_same_v<X, Three> ? 8 : 16 / (int)sizeof(X);
template <typename X, typename T> __device__ __forceinline__ void copy_chunk(const T *row, int c, int cols, X *to)
{
    if constexpr (std::is_same_v<X, Three>) {
        float f[8];
        widen<float>(ld_chunk(row, c, cols), f);
        widen<float>(ld_chunk(row, c + 4, cols), f + 4);
        put_three(to + c / GROUP * GROUP, c % GROUP, f);
    } else {
        *(u32x4 *)(to + c) = ld_chunk(row, c, cols);
    }
}

// Rows at multiples of 16 bytes for tensors that have none, or in three parts: zeros up to `ld`.
template <typename X, typename T>
__global__ __launch_bounds__(256) void kt_xent_align_kernel(const T *x, int64_t ldx, int cols, X *y, int64_t ld, int64_t rows)
{
    const int parts = (int)((ld + 64 * EACH<X> - 1) / (64 * EACH<X>));
    for (int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; n < rows * parts; n += (int64_t)gridDim.x * 4) {
        const int64_t row = n / parts;
        const int c = (int)(n % parts) * 64 * EACH<X> + (threadIdx.x & 63) * EACH<X>;
        if (c < ld) copy_chunk(x + row * ldx, c, cols, y + row * ld);
    }
}

// lse and loss from the parts' largest values and sums: 256 / TOKENS lanes for a token, each a stretch of the parts or (one token) every 256th.
template <typename I, int TOKENS>
__global__ __launch_bounds__(256) void kt_xent_join_kernel(const f32x2 *parts, int count, const float *hit, const I *targets, int tokens,
                                                           int vocab, float *loss, float *lse)
{
    constexpr int EACH = 256 / TOKENS, LEFT = TOKENS == 1 ? 4 : EACH;
    __shared__ f32x2 of[LEFT][TOKENS];
    const int i = threadIdx.x % TOKENS, w = threadIdx.x / TOKENS;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + i;
    const bool on = t < tokens && target_of(targets, (int)min(t, (int64_t)INT32_MAX), tokens, vocab) >= 0;
    float top = -INFINITY, sum = 0;
    auto add = [&](f32x2 p) {
        const float m = fmaxf(top, p[0]), base = m == -INFINITY ? 0.0f : m;
        sum = sum * __builtin_amdgcn_exp2f((top - base) * LOG2E) + p[1] * __builtin_amdgcn_exp2f((p[0] - base) * LOG2E);
        top = m;
    };
    if (on) {
        const int each = (count + EACH - 1) / EACH, a = TOKENS == 1 ? w : w * each, b = TOKENS == 1 ? count : min(count, a + each);
#pragma unroll 8
        for (int k = a; k < b; k += TOKENS == 1 ? EACH : 1) add(parts[(int64_t)k * tokens + t]);
    }
    if constexpr (TOKENS == 1) {
#pragma unroll
        for (int d = 32; d; d /= 2) add(f32x2{__shfl_xor(top, d), __shfl_xor(sum, d)});
        if ((threadIdx.x & 63) == 0) of[threadIdx.x / 64][0] = f32x2{top, sum};
    } else {
        of[w][i] = f32x2{top, sum};
    }
    __syncthreads();
    if (w || t >= tokens) return;
    for (int k = 1; k < LEFT; ++k) add(of[k][i]);
    // the loss not by way of lse, whose rounding a likely target's loss would be small beside
    const float rest = __builtin_amdgcn_logf(sum) * LN2, all = top + rest;
    loss[t] = on ? (top - hit[t]) + rest : 0.0f;
    if (lse) lse[t] = on ? all : 0.0f;
}

// Whether a token takes part; dloss or null: all with a target.  `top`: the largest finite dloss so far.
template <typename I> __device__ __forceinline__ bool takes_part(const I *targets, const float *dloss, int t, int tokens, int vocab, float &top)
{
    if (target_of(targets, t, tokens, vocab) < 0) return false;
    if (!dloss) return true;
    const float up = fabsf(dloss[t]);
    if (up < INFINITY) top = fmaxf(top, up);
    return up != 0.0f;
}

// How many of 1024 tokens do.
template <typename I>
__global__ __launch_bounds__(1024) void kt_xent_count_kernel(const I *targets, const float *dloss, int tokens, int vocab, int *counts, float *tops)
{
    __shared__ float most[16];
    __shared__ int mine[16];
    float top = 0;
    const uint64_t word = __ballot(takes_part(targets, dloss, blockIdx.x * 1024 + threadIdx.x, tokens, vocab, top));
    for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    if ((threadIdx.x & 63) == 0) {
        mine[threadIdx.x / 64] = __popcll(word);
        most[threadIdx.x / 64] = top;
    }
    __syncthreads();
    if (threadIdx.x) return;
    int n = 0;
    for (int w = 0; w < 16; ++w) {
        n += mine[w];
        top = fmaxf(top, most[w]);
    }
    counts[blockIdx.x] = n;
    tops[blockIdx.x] = top;
}

// The tokens that take part, in their order, and their number; the largest finite dloss of one.  A workgroup counts those before its own by itself, which takes
// one launch, or (`counts`, of 8193 tokens on) adds what others have counted: 16384 tokens take 20 us by themselves and 10 in two launches.
template <typename I>
__global__ __launch_bounds__(1024) void kt_xent_list_kernel(const I *targets, const float *dloss, int tokens, int vocab, const int *counts, const float *tops, int *map,
                                                            int *live, float *unit, int *goals)
{
    __shared__ int before[16], mine[16];
    __shared__ float most[16];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, first = blockIdx.x * 1024, t = first + threadIdx.x;
    int n = 0;
    float top = 0;
    if (counts) {
        for (int at = threadIdx.x; at < (int)blockIdx.x; at += 1024) {
            n += counts[at];
            top = fmaxf(top, tops[at]);
        }
    } else {
#pragma unroll 4
        for (int at = threadIdx.x; at < first; at += 1024) n += takes_part(targets, dloss, at, tokens, vocab, top);
    }
    const bool on = takes_part(targets, dloss, t, tokens, vocab, top);
    for (int d = 32; d; d /= 2) {
        n += __shfl_xor(n, d);
        top = fmaxf(top, __shfl_xor(top, d));
    }
    const uint64_t word = __ballot(on);
    if (lane == 0) {
        before[wave] = n;
        mine[wave] = __popcll(word);
        most[wave] = top;
    }
    __syncthreads();
    int at = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        at += before[w] + (w < wave ? mine[w] : 0);
        all += before[w] + mine[w];
    }
    if (on) {
        const int row = at + __popcll(word & ((1ull << lane) - 1));
        map[row] = t;
        if (goals) goals[row] = (int)targets[t];
    }
    if (threadIdx.x || blockIdx.x != gridDim.x - 1) return;
    *live = all;
    if (!unit) return;
    for (int w = 0; w < 16; ++w) top = fmaxf(top, most[w]);
    *unit = top > 0 ? top : 1.0f;
}

// Their rows of x one after another, zeros up to `ld`; where dx is given, zeros into its rows of the other tokens.
template <typename X, typename T, typename I>
__global__ __launch_bounds__(256) void kt_xent_gather_kernel(const T *x, int64_t ldx, int cols, X *y, int64_t ld, const int *map, const int *live,
                                                             const I *targets, const float *dloss, int tokens, int vocab, T *dx, int64_t lddx)
{
    const int parts = (int)((ld + 64 * EACH<X> - 1) / (64 * EACH<X>)), count = *live;
    for (int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; n < (int64_t)tokens * parts; n += (int64_t)gridDim.x * 4) {
        const int t = (int)(n / parts), c = (int)(n % parts) * 64 * EACH<X> + (threadIdx.x & 63) * EACH<X>;
        if (c >= ld) continue;
        if (t < count) copy_chunk(x + map[t] * ldx, c, cols, y + t * ld);
        if (dx && !(target_of(targets, t, tokens, vocab) >= 0 && dloss[t] != 0.0f)) {
#pragma unroll
            for (int k = 0; k < EACH<X>; k += VE<T>)
                if (c + k < cols) st_chunk(dx + t * lddx, c + k, cols, u32x4{0, 0, 0, 0});
        }
    }
}

// The sum of pieces of k, in their order; rows of the pieces `ldp` apart.  map, live, unit, rests: as Result has them.
template <typename G>
__global__ __launch_bounds__(256) void kt_xent_sum_kernel(const float *parts, int pieces, int64_t apart, int ldp, int rows, int cols, G *out, int64_t ld, const int *map,
                                                           const int *live, const float *unit, Rests rests)
{
    const int across = (cols + 3) / 4;
    if (live) rows = *live;
    const float of = unit ? *unit : 1.0f;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < (int64_t)rows * across; n += (int64_t)gridDim.x * 256) {
        const int64_t row = n / across;
        const int c = (int)(n % across) * 4;
        const float *p = parts + row * ldp + c;
        const int64_t to = (map ? map[row] : row) * ld;
        f32x4 s = *(const f32x4 *)p;
        for (int k = 1; k < pieces; ++k) s += *(const f32x4 *)(p + k * apart);
        if constexpr (sizeof(G) == 2) {
            if (rests.rest) {
                const G *w = static_cast<const G *>(rests.w) + rests.goals[row] * rests.ldw;
                for (int j = 0; j < 4; ++j)
                    if (c + j < cols) s[j] += rests.rest[row] * (float)w[c + j];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < cols) out[to + c + j] = (G)(s[j] * of);
    }
}

// ---- how the work is cut ---------------------------------------------------------------

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t over(int64_t n, int64_t by) { return (n + by - 1) / by; }

// How a product of m x n over k is cut: the tile's side, and pieces of k (at most `most`), whose sums a second kernel adds.
struct Cut {
    int side, pieces, piece;        // side 0: tiles of numbers in three parts
    int64_t m() const { return side ? side : Split::BM; }
    int64_t n() const { return side ? side : Split::BN; }
    int64_t part() const { return side ? side / 2 : Split::FM * 32; }       // rows of m that a wavefront has
};
// The least time of a model in us: a CU makes one workgroup's tile after the other, elements times steps of k at a rate that depends on the side (and a
// start and an end worth 128 steps); pieces cost a launch and their sums' way through memory.  Rates are what full chips reached (16384 x 8192 x 2048 in its three orders: tiles of 256 511
// to 555 us, of 128 600 to 650, of 64 850 to 1060; f32 4096 x 32768 x 768: 128 1578 to 1684, 64 1639 to 1829; in
// three parts 8192 x 50304 x 768 3000).  Both sides of a choice, us: f32
// 768 x 4096 over 32768 in 2 pieces (384 workgroups) 2024, in 4 (768) 1578; bf16 2048 x 1152 over 16384 in tiles of 64 206, of 128 in 3 pieces 122.
// A workgroup of 4 wavefronts that has a CU to itself waits for its loads with nothing beside it, `alone` times the rate.  Without that and with it, gradients: 1024 tokens of
// 50304 x 768 bf16 382 and 352 (dx in twice the pieces), 4000 of 300 x 768 46.6 and 42.9, f32 92 of 50304 x 1024 422 and 383, 1000 of 1000 x 768 91.7 and 83.9.
Cut cut_of(kt_dtype dt, bool three, int64_t m, int64_t n, int64_t k, int64_t most)
{
    Cut best{three ? 0 : 64, 1, (int)up(k < 1 ? 1 : k, 64)};
    double least = 1e300;
    for (int side : {0, 256, 128, 64}) {
        if (three != (side == 0) || (side == 256 && dt == KT_F32)) continue;
        const double rate = three ? 4.0e5 : dt == KT_F32 ? (side == 128 ? 2.5e5 : 2.3e5) : side == 256 ? 2.0e6 : side == 128 ? 1.75e6 : 1.15e6;
        const double alone = side == 64 ? 0.6 : side == 128 ? 0.7 : 1;
        const Cut c{side, 1, 0};
        const int64_t tiles = over(m, c.m()) * over(n, c.n());
        for (int64_t p = 1; p <= most && (p == 1 || p * 128 <= k); ++p) {
            const int64_t piece = up(over(k < 1 ? 1 : k, p), 64), count = over(k < 1 ? 1 : k, piece);
            if (count != p) continue;
            const double t = (double)over(tiles * p, 256) * c.m() * c.n() * (double)(piece + 128) / (tiles * p <= 256 ? alone * rate : rate) + (p > 1 ? 4 + (double)m * n * 8 * p / 5.5e6 : 0);
            if (t < least) {
                least = t;
                best = Cut{side, (int)p, (int)piece};
            }
        }
    }
    return best;
}
constexpr int64_t MOST_PIECES = 64;

// Whether loads of 16 bytes can take a matrix as it is: rows at multiples of 16 bytes, offsets within a tile of 31 bits.
template <typename T> bool plain(const T *p, int64_t ld, int64_t width)
{
    return rows_of_16(p, ld) && width % VE<T> == 0 && ld * (int64_t)sizeof(T) <= 1 << 22;
}

// Whether kt_xent_few_kernel makes the logits: up to 16 tokens, and up to 32 where tiles would need a copy of the weight or have little to do.  us, forward
// pass: 30 tokens of 50304 x 2048 bf16 85, in tiles 55; of 50304 x 1001 f32 93 and 150; of 5003 x 768 bf16 9.9 and 11.9; 12 of 50304 x 2048 56 and 53.
bool few_tokens(kt_dtype dt, int64_t tokens, int64_t vocab, int64_t width)
{
    return tokens <= 16 || (tokens <= 32 && (width * (dt == KT_F32 ? 4 : 2) % 16 || vocab * width < 1 << 25));
}

// Whether f32 products are made of numbers in three parts: where the copies into parts cost little beside them and tiles of 256 x 128 keep the chip busy.  The
// same in both passes, so that their logits have the same bits.  us, f32 instructions and parts: 8192 tokens of 50304 x 768 4850 and 3010 forward and
// 15300 and 10030 backward, 1024 of 5003 x 1001 115 and 90, 328 and 233, 512 of 5003 x 1024 65 and 89, 188 and 176; but 2048 of 1000 x 4096 181 and 263, 471
// and 451, 1024 of 1000 x 768 28 and 68, 92 and 125, 100 of 50304 x 768 111 and 150, 329 and 334.
bool in_three(kt_dtype dt, int64_t tokens, int64_t vocab, int64_t width)
{
    return dt == KT_F32 && width >= 128 && tokens >= 256 && over(vocab, Split::BM) * over(tokens, Split::BN) >= 80;
}

// What a call needs of the workspace, and its cut.  Matrices that loads of 16 bytes cannot take as they are are copied to rows of a multiple of 16 bytes first
// (the weight up to 128 MiB of it at a time; 512 in three parts, whose tiles of 256 rows would else be few: gradients of 300 tokens of
// 50304 x 4096 4509 and 2985 us), which costs their bytes twice more: 4099 tokens of 5003 x 1001 8 of 137 us.
struct Plan {
    bool three;                     // operands in three parts
    int64_t es, wide;               // bytes of an operand's element; elements to a row of a copy
    int64_t copy;                   // rows of the weight copied at a time
    int64_t most, piece;            // rows of the vocabulary in a piece: with the weight as it is; with copies
    Cut z;                          // of the logits of the whole vocabulary
    int64_t slopes;                 // wavefronts that share a token's logits then
    bool few;                       // kt_xent_few_kernel makes them
    int64_t ldp;                    // backward: elements to a row of sums
    Cut kx;                         // of dx over a piece of the vocabulary
    bool list;                      // whether the tokens that take part are listed
    int64_t goals, rest;            // bf16, backward
    int64_t x, w, parts, hit, others, likely, ids, table, dz, map, live, acc, sums, bytes;      // where in the workspace
};
// Wavefronts that share a token's logits of `rows` rows of the vocabulary.
int64_t sharing(bool few, const Cut &z, int64_t rows) { return few ? over(rows, 16) : over(rows, z.m()) * (z.m() / z.part()); }
int64_t at_most(int64_t a, int64_t b) { return a < b ? a : b; }
// Rows of a multiple of 256 that keep rows * of below `most`.
int64_t rows_in(int64_t most, int64_t of, int64_t vocab)
{
    int64_t r = most / (of < 1 ? 1 : of) / 256 * 256;
    if (r < 256) r = 256;
    return at_most(r, up(vocab, 256));
}
Plan plan_of(kt_dtype dt, int64_t tokens, int64_t vocab, int64_t width, bool bwd)
{
    Plan p{};
    p.three = in_three(dt, tokens, vocab, width);
    p.es = p.three ? sizeof(Three) : dt == KT_F32 ? 4 : 2;
    p.wide = up(width, 64);
    p.copy = rows_in((p.three ? 512 : 128) << 20, p.wide * p.es, vocab);
    // backward: dz of up to 2^27 elements, 256 MiB of bf16, what the last-level cache holds; forward: a launch of up to 2^20 tiles of 256
    p.most = rows_in(bwd ? 1ll << (p.three ? 26 : 27) : 1ll << 36, tokens, vocab);
    if (bwd) p.most = at_most(p.most, 1 << 18);
    p.piece = at_most(p.most, p.copy);
    p.z = cut_of(dt, p.three, vocab, tokens, width, 1);
    p.ldp = up(width, 16);
    auto take = [&](int64_t bytes) {
        const int64_t from = p.bytes;
        p.bytes += up(bytes, 256);
        return from;
    };
    const bool few = p.few = few_tokens(dt, tokens, vocab, width);
    p.x = take(!bwd && few ? 0 : tokens * p.wide * p.es);
    p.w = take(!bwd && few ? 0 : p.piece * p.wide * p.es);
    // a list and a copy of x cost some 6 us and its bytes twice: worth while for the forward pass from some 100 us on
    p.list = bwd || p.three || (double)tokens * vocab * width * (dt == KT_F32 ? 8 : 1) > 5e10;
    p.map = take(p.list ? tokens * 4 : 0);
    p.live = take(p.list ? 8 + over(tokens, 1024) * 8 : 0);
    p.slopes = sharing(few, p.z, vocab);
    if (!bwd) {
        p.parts = take(p.slopes * tokens * 8);
        p.hit = take(tokens * 4);
        return p;
    }
    // rows of a piece of the vocabulary, whole ones and the last, with the weight as it is and with copies
    const int64_t sizes[] = {at_most(p.most, vocab), at_most(p.piece, vocab), vocab % p.most, vocab % p.piece};
    if (dt == KT_F32) {
        int64_t most = 0;
        for (int64_t rows : sizes) {
            const int64_t n = rows ? sharing(few, cut_of(dt, p.three, rows, tokens, width, 1), rows) : 0;
            if (n > most) most = n;
        }
        p.others = take(most * tokens * 4);
        if (p.piece < vocab) {
            p.likely = take(tokens * 8);
            p.ids = take(tokens * 4);
            p.table = take(kt_embedding_bwd_ws(tokens, vocab, width));
        }
    }
    if (dt == KT_BF16) {
        p.goals = take(tokens * 4);
        p.rest = take(tokens * 4);
    }
    p.dz = take(tokens * p.most * p.es);
    p.kx = cut_of(dt, p.three, width, tokens, at_most(p.most, vocab), MOST_PIECES);
    if (p.piece < vocab) p.acc = take(p.kx.pieces * over(width, p.kx.m()) * over(tokens, p.kx.n()) * p.kx.m() * p.kx.n() * 4);
    // dx cut over the vocabulary, and the weight's gradient cut over the tokens: whichever takes more
    int64_t most = p.kx.pieces > 1 ? p.kx.pieces * tokens : 0;
    for (int64_t rows : sizes) {
        if (rows == 0) continue;
        const Cut k = cut_of(dt, p.three, width, rows, tokens, MOST_PIECES);
        if (k.pieces > 1 && k.pieces * rows > most) most = k.pieces * rows;
    }
    p.sums = take(most * p.ldp * 4);
    return p;
}

template <typename T, typename S, bool AA, bool BA, typename E>
int launch_tiles(const Operand<T> &a, int64_t m, const Operand<T> &b, int64_t n, int64_t steps, const Cut &k, const int *live, const E &e, hipStream_t s)
{
    constexpr int LDS = S::SLOTS * (S::BM + S::BN) * ROW;
    const auto kernel = kt_xent_product_kernel<T, S, AA, BA, E>;
    if (LDS > 65536) {
        const hipError_t e1 = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e1 != hipSuccess) return (int)e1;
    }
    const int64_t mt = over(m, S::BM), nt = over(n, S::BN);
    kernel<<<dim3((unsigned)(mt * nt), (unsigned)k.pieces), S::BLOCK, LDS, s>>>(a, b, (int)steps, k.piece, live, (int)mt, (int)nt, e);
    return (int)hipGetLastError();
}
// The product of A [m x steps] and B [n x steps].
template <typename T, bool AA, bool BA, typename E>
int product(const Cut &k, const Operand<T> &a, int64_t m, const Operand<T> &b, int64_t n, int64_t steps, const int *live, const E &e, hipStream_t s)
{
    if constexpr (std::is_same_v<T, Three>) {
        constexpr int LDS = 2 * Split::SLOT;
        const auto kernel = kt_xent_three_kernel<AA, BA, E>;
        const hipError_t e1 = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e1 != hipSuccess) return (int)e1;
        const int64_t mt = over(m, Split::BM), nt = over(n, Split::BN);
        kernel<<<dim3((unsigned)(mt * nt), (unsigned)k.pieces), Split::BLOCK, LDS, s>>>(a, b, (int)steps, k.piece, live, (int)mt, (int)nt, e);
        return (int)hipGetLastError();
    } else {
        if constexpr (sizeof(T) == 2) {
            if (k.side == 256) return launch_tiles<T, Big, AA, BA>(a, m, b, n, steps, k, live, e, s);
        }
        if (k.side == 128) return launch_tiles<T, Mid, AA, BA>(a, m, b, n, steps, k, live, e, s);
        return launch_tiles<T, Small, AA, BA>(a, m, b, n, steps, k, live, e, s);
    }
}

#define KT_GO(call)                    \
    do {                               \
        const int go_ = (call);        \
        if (go_) return go_;           \
    } while (0)

template <typename T, typename E> int few(const T *w, int64_t ldw, int64_t rows, const T *x, int64_t ldx, int64_t tokens, int64_t width, const E &e, hipStream_t s)
{
    const unsigned blocks = (unsigned)over(rows, 16);
    if (tokens <= 16) kt_xent_few_kernel<T, 1, E><<<blocks, 64, 0, s>>>(w, ldw, (int)rows, x, ldx, (int)tokens, (int)width, e);
    else kt_xent_few_kernel<T, 2, E><<<blocks, 64, 0, s>>>(w, ldw, (int)rows, x, ldx, (int)tokens, (int)width, e);
    return (int)hipGetLastError();
}

// x or rows of w as the products take them: as they are, or copied.
template <typename X, typename T>
int aligned_rows(bool as_is, const T *x, int64_t ldx, int64_t width, int64_t rows, X *copy, int64_t wide, Operand<X> *to, hipStream_t s)
{
    to->count = (int)rows;
    if constexpr (std::is_same_v<X, T>) {
        if (as_is) {
            to->p = x;
            to->ld = ldx;
            return 0;
        }
    }
    to->p = copy;
    to->ld = wide;
    if (rows == 0) return 0;
    const int64_t blocks = over(rows * over(wide, 64 * EACH<X>), 4);
    kt_xent_align_kernel<X, T><<<(unsigned)at_most(blocks, 1 << 20), 256, 0, s>>>(x, ldx, (int)width, copy, wide, rows);
    return (int)hipGetLastError();
}

// The list of the tokens that take part and their rows of x; zeros in dx's rows of the others.
template <typename X, typename T, typename I>
int list(const T *x, int64_t ldx, int64_t width, const I *targets, const float *dloss, int64_t tokens, int64_t vocab, X *copy, int64_t wide, int *map,
         int *live, float *unit, T *dx, int64_t lddx, int *goals, hipStream_t s)
{
    const unsigned groups = (unsigned)over(tokens, 1024);
    int *const counts = groups > 8 ? live + 2 : nullptr;
    float *const tops = (float *)(live + 2 + groups);
    if (counts) kt_xent_count_kernel<I><<<groups, 1024, 0, s>>>(targets, dloss, (int)tokens, (int)vocab, counts, tops);
    KT_GO((int)hipGetLastError());
    kt_xent_list_kernel<I><<<groups, 1024, 0, s>>>(targets, dloss, (int)tokens, (int)vocab, counts, tops, map, live, unit, goals);
    KT_GO((int)hipGetLastError());
    const int64_t blocks = over(tokens * over(wide, 64 * EACH<X>), 4);
    kt_xent_gather_kernel<X, T, I><<<(unsigned)at_most(blocks, 1 << 20), 256, 0, s>>>(x, ldx, (int)width, copy, wide, map, live, targets, dloss, (int)tokens, (int)vocab, dx, lddx);
    return (int)hipGetLastError();
}

// X: the operands' type.
template <typename X, typename T, typename I>
int fwd(const Plan &p, kt_dtype dt, int64_t tokens, int64_t vocab, int64_t width, const T *x, int64_t ldx, const T *w, int64_t ldw, const I *targets, float *loss,
        float *lse, char *ws, hipStream_t s)
{
    f32x2 *parts = (f32x2 *)(ws + p.parts);
    int *const map = p.list ? (int *)(ws + p.map) : nullptr, *const live = p.list ? (int *)(ws + p.live) : nullptr;
    float *hit = (float *)(ws + p.hit);
    const bool w_as_is = std::is_same_v<X, T> && plain(w, ldw, width), by_few = few_tokens(dt, tokens, vocab, width);
    X *const copy = (X *)(ws + p.x);
    Operand<X> a, b;
    const int count = (int)p.slopes;
    if (by_few) {
        const Stats<I> e{parts, hit, targets, nullptr, nullptr, (int)tokens, (int)vocab, 0, (int)vocab, 0};
        KT_GO(few(w, ldw, vocab, x, ldx, tokens, width, e, s));
    } else if (p.list) {
        KT_GO((list<X, T, I>(x, ldx, width, targets, nullptr, tokens, vocab, copy, p.wide, map, live, nullptr, nullptr, 0, nullptr, s)));
        b = Operand<X>{copy, p.wide, (int)tokens};
    } else {
        KT_GO((aligned_rows<X, T>(plain(x, ldx, width), x, ldx, width, tokens, copy, p.wide, &b, s)));
    }
    for (int64_t v = by_few ? vocab : 0, rows; v < vocab; v += rows) {
        rows = at_most(w_as_is ? p.most : p.piece, vocab - v);
        KT_GO((aligned_rows<X, T>(w_as_is, w + v * ldw, ldw, width, rows, (X *)(ws + p.w), p.wide, &a, s)));
        const Stats<I> e{parts, hit, targets, map, live, (int)tokens, (int)vocab, (int)v, (int)(v + rows), (int)(v / p.z.part())};
        KT_GO((product<X, true, true>(p.z, a, rows, b, tokens, width, live, e, s)));
    }
    if (tokens >= 512) kt_xent_join_kernel<I, 32><<<(unsigned)over(tokens, 32), 256, 0, s>>>(parts, count, hit, targets, (int)tokens, (int)vocab, loss, lse);
    else kt_xent_join_kernel<I, 1><<<(unsigned)tokens, 256, 0, s>>>(parts, count, hit, targets, (int)tokens, (int)vocab, loss, lse);
    return (int)hipGetLastError();
}

template <typename G> int sum(const float *parts, const Cut &k, int64_t apart, int64_t ldp, int64_t rows, int64_t cols, G *out, int64_t ld, const int *map, const int *live,
                              const float *unit, const Rests &rests, hipStream_t s)
{
    const int64_t blocks = over(rows * over(cols, 4), 256);
    kt_xent_sum_kernel<G><<<(unsigned)at_most(blocks, 1 << 20), 256, 0, s>>>(parts, k.pieces, apart, (int)ldp, (int)rows, (int)cols, out, ld, map, live, unit, rests);
    return (int)hipGetLastError();
}

template <typename X, typename T, typename I>
int bwd(const Plan &p, kt_dtype dt, int64_t tokens, int64_t vocab, int64_t width, const float *dloss, const T *x, int64_t ldx, const T *w, int64_t ldw,
        const I *targets, const float *lse, T *dx, int64_t lddx, T *dw, int64_t lddw, char *ws, hipStream_t s)
{
    int *const map = (int *)(ws + p.map), *const live = (int *)(ws + p.live);
    X *dz = (X *)(ws + p.dz);
    float *acc = (float *)(ws + p.acc), *sums = (float *)(ws + p.sums);
    const bool w_as_is = std::is_same_v<X, T> && plain(w, ldw, width);
    constexpr int UNIT = std::is_same_v<X, Three> ? GROUP : VE<T>;
    // bf16: dz in units of the largest dloss, so that a mean's 1 / tokens, the same share of every token, is not rounded with it
    float *const unit = tokens && sizeof(T) == 2 ? (float *)live + 1 : nullptr;
    const int64_t cols = up(width, UNIT);               // of an operand: what a copy has past the width is zeros
    const int64_t piece = w_as_is ? p.most : p.piece;
    const bool several = piece < vocab;
    float *const others = sizeof(T) == 4 ? (float *)(ws + p.others) : nullptr, *const likely = (float *)(ws + p.likely);
    X *const copy = (X *)(ws + p.x);
    constexpr bool HALVES = sizeof(T) == 2;
    int *const goals = HALVES ? (int *)(ws + p.goals) : nullptr;
    float *const rest = HALVES ? (float *)(ws + p.rest) : nullptr;
    const Rests none{}, of_dx{rest, goals, 0, w, ldw};
    Operand<X> a;
    const Operand<X> b{copy, p.wide, (int)tokens};
    if (tokens) KT_GO((list<X, T, I>(x, ldx, width, targets, dloss, tokens, vocab, copy, p.wide, map, live, unit, dx, lddx, goals, s)));
    for (int64_t v = 0, rows; v < vocab; v += rows) {
        rows = at_most(piece, vocab - v);
        if (tokens) {
            KT_GO((aligned_rows<X, T>(w_as_is, w + v * ldw, ldw, width, rows, (X *)(ws + p.w), p.wide, &a, s)));
            const Cut z = cut_of(dt, p.three, rows, tokens, width, 1);
            const int parts = (int)sharing(p.few, z, rows);
            const Slope<X, I> e{dz, p.most, lse, dloss, unit, others, targets, map, live, (int)tokens, (int)vocab, (int)v, (int)(v + rows), parts, rest};
            bool made = false;
            if constexpr (std::is_same_v<X, T>) {
                made = p.few;
                if (made) KT_GO(few(a.p, a.ld, rows, (const T *)copy, p.wide, tokens, width, e, s));
            }
            if (!made) KT_GO((product<X, true, true>(z, a, rows, b, tokens, width, live, e, s)));
            if constexpr (sizeof(T) == 4) {
                const unsigned blocks = (unsigned)over(tokens, 4);
                if (!several) kt_xent_target_kernel<X, I><<<blocks, 256, 0, s>>>(dz, p.most, others, parts, dloss, targets, map, live);
                else kt_xent_others_kernel<X, I><<<blocks, 256, 0, s>>>(dz, p.most, others, parts, targets, map, live, (int)v, (int)(v + rows), likely, likely + tokens);
                KT_GO((int)hipGetLastError());
            }
        }
        if (dx && tokens) {
            const Operand<X> wide{a.p, a.ld, (int)cols}, slope{dz, p.most, (int)tokens};
            const bool first = v == 0, last = v + rows == vocab;
            const Cut k{p.kx.side, p.kx.pieces, (int)up(over(rows, p.kx.pieces), 64)};
            if (!last) {
                const Carry e{acc, first};
                KT_GO((product<X, false, true>(k, wide, width, slope, tokens, rows, live, e, s)));
            } else if (k.pieces == 1) {
                const Result<T> e{dx, lddx, 0, first ? nullptr : acc, map, live, unit, (int)tokens, (int)width, of_dx};
                KT_GO((product<X, false, true>(k, wide, width, slope, tokens, rows, live, e, s)));
            } else {
                const int64_t apart = tokens * p.ldp;
                const Result<float> e{sums, p.ldp, apart, first ? nullptr : acc, nullptr, live, nullptr, (int)tokens, (int)p.ldp, none};
                KT_GO((product<X, false, true>(k, wide, width, slope, tokens, rows, live, e, s)));
                KT_GO(sum(sums, k, apart, p.ldp, tokens, width, dx, lddx, map, live, unit, of_dx, s));
            }
        }
        if (dw) {
            const Operand<X> wide{b.p, b.ld, (int)cols}, slope{dz, p.most, (int)up(rows, UNIT)};
            const Cut k = cut_of(dt, p.three, width, rows, tokens, MOST_PIECES);
            const Rests of_dw{rest, goals, (int)v, nullptr, 0};
            if (k.pieces == 1) {
                const Result<T, HALVES> e{dw + v * lddw, lddw, 0, nullptr, nullptr, nullptr, unit, (int)rows, (int)width, of_dw};
                KT_GO((product<X, false, false>(k, wide, width, slope, rows, tokens, tokens ? live : nullptr, e, s)));
            } else {
                const Result<float, HALVES> e{sums, p.ldp, rows * p.ldp, nullptr, nullptr, nullptr, nullptr, (int)rows, (int)p.ldp, of_dw};
                KT_GO((product<X, false, false>(k, wide, width, slope, rows, tokens, tokens ? live : nullptr, e, s)));
                KT_GO(sum(sums, k, rows * p.ldp, p.ldp, rows, width, dw + v * lddw, lddw, nullptr, nullptr, unit, none, s));
            }
        }
    }
    if constexpr (sizeof(T) == 4) {
        if (several && tokens) {
            // all products are made, so the copy of x is free for the rows that dw gets
            int *const ids = dw ? (int *)(ws + p.ids) : nullptr;
            const int64_t blocks = over(tokens * over(width, 256), 4);
            kt_xent_likely_kernel<I><<<(unsigned)at_most(blocks, 1 << 20), 256, 0, s>>>(likely, likely + tokens, dloss, targets, map, live, (int)tokens, (int)width, x, ldx, w, ldw,
                                                                                      dx, lddx, (float *)copy, p.wide, ids);
            KT_GO((int)hipGetLastError());
            if (dw) return kt_launch_embedding_bwd(KT_F32, KT_F32, KT_I32, tokens, (int)vocab, (int)width, ids, copy, p.wide, 1.0f, dw, lddw, true, ws + p.table, s);
        }
    }
    return 0;
}

template <typename F> int by_types(kt_dtype dt, kt_index it, F f)
{
    auto index = [&](auto t) { return it == KT_I32 ? f(t, int32_t()) : f(t, int64_t()); };
    return dt == KT_F32 ? index(float()) : index(bf16());
}

}  // namespace

int64_t kt_linear_xent_ws(kt_dtype dt, int64_t tokens, int64_t vocab, int64_t width, bool bwd) { return plan_of(dt, tokens, vocab, width, bwd).bytes; }

int kt_launch_linear_xent_fwd(kt_dtype dt, kt_index it, int64_t tokens, int64_t vocab, int64_t width, const void *x, int64_t ldx, const void *w,
                              int64_t ldw, const void *targets, float *loss, float *lse, void *ws, void *stream)
{
    return by_types(dt, it, [&](auto t, auto i) {
        typedef decltype(t) T;
        typedef decltype(i) I;
        const Plan p = plan_of(dt, tokens, vocab, width, false);
        if constexpr (sizeof(T) == 4) {
            if (p.three) return fwd<Three, T, I>(p, dt, tokens, vocab, width, (const T *)x, ldx, (const T *)w, ldw, (const I *)targets, loss, lse, (char *)ws, (hipStream_t)stream);
        }
        return fwd<T, T, I>(p, dt, tokens, vocab, width, (const T *)x, ldx, (const T *)w, ldw, (const I *)targets, loss, lse, (char *)ws, (hipStream_t)stream);
    });
}

int kt_launch_linear_xent_bwd(kt_dtype dt, kt_index it, int64_t tokens, int64_t vocab, int64_t width, const float *dloss, const void *x, int64_t ldx,
                              const void *w, int64_t ldw, const void *targets, const float *lse, void *dx, int64_t lddx, void *dw, int64_t lddw,
                              void *ws, void *stream)
{
    return by_types(dt, it, [&](auto t, auto i) {
        typedef decltype(t) T;
        typedef decltype(i) I;
        const Plan p = plan_of(dt, tokens, vocab, width, true);
        if constexpr (sizeof(T) == 4) {
            if (p.three)
                return bwd<Three, T, I>(p, dt, tokens, vocab, width, dloss, (const T *)x, ldx, (const T *)w, ldw, (const I *)targets, lse, (T *)dx, lddx, (T *)dw, lddw, (char *)ws, (hipStream_t)stream);
        }
        return bwd<T, T, I>(p, dt, tokens, vocab, width, dloss, (const T *)x, ldx, (const T *)w, ldw, (const I *)targets, lse, (T *)dx, lddx, (T *)dw, lddw, (char *)ws, (hipStream_t)stream);
    });
}
