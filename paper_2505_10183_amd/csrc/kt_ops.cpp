// C entry points of the operators (kt_ops.h): argument checks on the host, then launches.  Nothing here allocates, uploads or
// waits, and nothing throws.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstddef>

#include "kt_ops_internal.h"

namespace {

bool is_type(kt_dtype t) { return t == KT_F32 || t == KT_BF16; }
int64_t size_of(kt_dtype t) { return t == KT_F32 ? 4 : 2; }

kt_status bad(const char *who, const char *what)
{
    kt_set_error("%s: %s", who, what);
    return KT_EINVAL;
}
kt_status unsupported(const char *who, const char *what)
{
    kt_set_error("%s: %s", who, what);
    return KT_EUNSUPPORTED;
}
kt_status aligned(const char *who, const char *name, const void *p, int64_t to)
{
    if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0) return KT_OK;
    kt_set_error("%s: %s is not aligned to %d bytes", who, name, (int)to);
    return KT_EALIGN;
}
kt_status launched(const char *who, int e)
{
    if (e == 0) return KT_OK;
    kt_set_error("%s: launch: %s", who, hipGetErrorString((hipError_t)e));
    return KT_EHIP;
}

// A matrix in memory; `row` and `ld` in bytes.
struct Block {
    const char *name;
    const void *p;
    int64_t rows, row, ld;
};
Block matrix(const char *name, const void *p, kt_dtype t, int64_t rows, int64_t cols, int64_t ld)
{
    return Block{name, p, rows, cols * size_of(t), ld * size_of(t)};
}
Block flat(const char *name, const void *p, int64_t bytes) { return Block{name, p, 1, bytes, bytes}; }

// Whether two matrices share a byte.  Columns of one buffer (equal distances between rows) may lie side by side.
bool overlap(const Block &a, const Block &b)
{
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.row < 1 || b.row < 1) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    if (a0 + (uintptr_t)((a.rows - 1) * a.ld + a.row) <= b0 || b0 + (uintptr_t)((b.rows - 1) * b.ld + b.row) <= a0) return false;
    if (a.rows == 1 || b.rows == 1 || a.ld != b.ld) return true;
    const int64_t d = b0 >= a0 ? (int64_t)((b0 - a0) % (uintptr_t)a.ld) : (a.ld - (int64_t)((a0 - b0) % (uintptr_t)a.ld)) % a.ld;
    return d < a.row || d + b.row > a.ld;
}
kt_status apart(const char *who, const Block &out, const Block &other)
{
    if (!overlap(out, other)) return KT_OK;
    kt_set_error("%s: %s overlaps %s", who, out.name, other.name);
    return KT_EINVAL;
}
// The same, for an output that may be the other matrix itself.
kt_status apart_or_same(const char *who, const Block &out, const Block &other)
{
    if (out.p == other.p && (out.ld == other.ld || out.rows <= 1)) return KT_OK;
    return apart(who, out, other);
}

// rows x cols with rows `ld` apart can be addressed, and so can what a checkpoint of it takes.
bool sizes(int64_t rows, int64_t cols, int64_t ld)
{
    const int64_t most = INT64_MAX / 16;
    if (rows < 0 || cols < 1 || ld < cols || ld > most) return false;
    const int64_t eight = kt_act8_groups(cols) * KT_ACT8_GROUP;
    return rows == 0 || (ld > eight ? ld : eight) <= most / rows;
}

#define KT_TRY(call)                        \
    do {                                    \
        const kt_status st_ = (call);       \
        if (st_ != KT_OK) return st_;       \
    } while (0)

}  // namespace

extern "C" kt_status kt_layernorm_fwd(kt_dtype dt, kt_dtype pdt, int64_t rows, int64_t cols, const void *x, int64_t ldx,
                                      const void *gamma, const void *beta, float eps, void *y, int64_t ldy, float *mean,
                                      float *rstd, int8_t *y8, uint8_t *e8, void *stream)
{
    const char *who = "kt_layernorm_fwd";
    if (!is_type(dt) || !is_type(pdt)) return bad(who, "unknown element type");
    if (!sizes(rows, cols, ldx) || !sizes(rows, cols, ldy)) return bad(who, "rows >= 0, cols >= 1 and ld >= cols are needed");
    if (cols > KT_LAYERNORM_MAX_COLS) return unsupported(who, "more than KT_LAYERNORM_MAX_COLS columns");
    if (!(eps >= 0.0f) || std::isinf(eps)) return bad(who, "eps must be finite and not negative");
    if (!gamma || (rows && (!x || !y))) return bad(who, "NULL x, gamma or y");
    if (!mean != !rstd) return bad(who, "mean and rstd go together");
    if (!y8 != !e8) return bad(who, "y8 and e8 go together");
    KT_TRY(aligned(who, "x", x, size_of(dt)));
    KT_TRY(aligned(who, "y", y, size_of(dt)));
    KT_TRY(aligned(who, "gamma", gamma, size_of(pdt)));
    KT_TRY(aligned(who, "beta", beta, size_of(pdt)));
    KT_TRY(aligned(who, "mean", mean, 4));
    KT_TRY(aligned(who, "rstd", rstd, 4));
    KT_TRY(aligned(who, "y8", y8, 16));
    const int64_t G = kt_act8_groups(cols);
    const Block in = matrix("x", x, dt, rows, cols, ldx), out = matrix("y", y, dt, rows, cols, ldy);
    const Block outs[] = {out, flat("mean", mean, rows * 4), flat("rstd", rstd, rows * 4),
                          flat("y8", y8, rows * G * KT_ACT8_GROUP), flat("e8", e8, rows * G)};
    const Block ins[] = {flat("gamma", gamma, cols * size_of(pdt)), flat("beta", beta, cols * size_of(pdt))};
    KT_TRY(apart_or_same(who, out, in));
    for (size_t i = 0; i < sizeof outs / sizeof *outs; ++i) {
        if (i) KT_TRY(apart(who, outs[i], in));
        for (const Block &b : ins) KT_TRY(apart(who, outs[i], b));
        for (size_t j = 0; j < i; ++j) KT_TRY(apart(who, outs[i], outs[j]));
    }
    if (rows == 0) return KT_OK;
    return launched(who, kt_launch_layernorm_fwd(dt, pdt, rows, (int)cols, x, ldx, gamma, beta, eps, y, ldy, mean, rstd, y8, e8, stream));
}

extern "C" kt_status kt_layernorm_bwd(kt_dtype dt, kt_dtype pdt, int64_t rows, int64_t cols, const void *dy, int64_t lddy,
                                      const void *x, int64_t ldx, const int8_t *x8, const uint8_t *e8, const void *gamma,
                                      const float *mean, const float *rstd, void *dx, int64_t lddx, void *dgamma,
                                      void *dbeta, void *ws, int64_t ws_bytes, void *stream)
{
    const char *who = "kt_layernorm_bwd";
    if (!is_type(dt) || !is_type(pdt)) return bad(who, "unknown element type");
    const bool eight = !x && (x8 || e8);
    if (eight) ldx = cols;
    if (!sizes(rows, cols, lddy) || !sizes(rows, cols, ldx) || !sizes(rows, cols, lddx))
        return bad(who, "rows >= 0, cols >= 1 and ld >= cols are needed");
    if (cols > KT_LAYERNORM_MAX_COLS) return unsupported(who, "more than KT_LAYERNORM_MAX_COLS columns");
    if (!gamma || !dgamma || (rows && (!dy || !mean || !rstd || !dx))) return bad(who, "NULL dy, gamma, mean, rstd, dx or dgamma");
    if (rows && (x ? (x8 || e8) : (!x8 || !e8))) return bad(who, "either x or both x8 and e8 are needed");
    const int64_t need = kt_layernorm_bwd_workspace(rows, cols);
    if (need && (!ws || ws_bytes < need)) return bad(who, "the workspace is smaller than kt_layernorm_bwd_workspace says");
    KT_TRY(aligned(who, "dy", dy, size_of(dt)));
    KT_TRY(aligned(who, "x", x, size_of(dt)));
    KT_TRY(aligned(who, "dx", dx, size_of(dt)));
    KT_TRY(aligned(who, "x8", x8, 16));
    KT_TRY(aligned(who, "gamma", gamma, size_of(pdt)));
    KT_TRY(aligned(who, "dgamma", dgamma, size_of(pdt)));
    KT_TRY(aligned(who, "dbeta", dbeta, size_of(pdt)));
    KT_TRY(aligned(who, "mean", mean, 4));
    KT_TRY(aligned(who, "rstd", rstd, 4));
    KT_TRY(aligned(who, "ws", ws, 16));
    const int64_t G = kt_act8_groups(cols), par = cols * size_of(pdt);
    const Block out = matrix("dx", dx, dt, rows, cols, lddx);
    const Block wide[] = {matrix("dy", dy, dt, rows, cols, lddy), matrix("x", x, dt, rows, cols, ldx)};
    const Block outs[] = {out, flat("dgamma", dgamma, par), flat("dbeta", dbeta, par), flat("ws", ws, need)};
    const Block ins[] = {flat("x8", x8, rows * G * KT_ACT8_GROUP), flat("e8", e8, rows * G), flat("gamma", gamma, par),
                         flat("mean", mean, rows * 4), flat("rstd", rstd, rows * 4)};
    for (const Block &b : wide) KT_TRY(apart_or_same(who, out, b));
    for (size_t i = 0; i < sizeof outs / sizeof *outs; ++i) {
        if (i)
            for (const Block &b : wide) KT_TRY(apart(who, outs[i], b));
        for (const Block &b : ins) KT_TRY(apart(who, outs[i], b));
        for (size_t j = 0; j < i; ++j) KT_TRY(apart(who, outs[i], outs[j]));
    }
    return launched(who, kt_launch_layernorm_bwd(dt, pdt, rows, (int)cols, dy, lddy, x, ldx, x8, e8, gamma, mean, rstd, dx, lddx,
                                                 dgamma, dbeta, (float *)ws, stream));
}

// Columns are 31-bit numbers in the kernels.
static const int64_t MOST_ACT8_COLS = 1 << 30;

extern "C" kt_status kt_act8_save(kt_dtype dt, int64_t rows, int64_t cols, const void *x, int64_t ldx, int8_t *q, uint8_t *e,
                                  void *stream)
{
    const char *who = "kt_act8_save";
    if (!is_type(dt)) return bad(who, "unknown element type");
    if (!sizes(rows, cols, ldx)) return bad(who, "rows >= 0, cols >= 1 and ld >= cols are needed");
    if (cols > MOST_ACT8_COLS) return unsupported(who, "more than 2^30 columns");
    if (rows == 0) return KT_OK;
    if (!x || !q || !e) return bad(who, "NULL x, q or e");
    KT_TRY(aligned(who, "x", x, size_of(dt)));
    KT_TRY(aligned(who, "q", q, 16));
    const int64_t G = kt_act8_groups(cols);
    const Block in = matrix("x", x, dt, rows, cols, ldx), b = flat("q", q, rows * G * KT_ACT8_GROUP), s = flat("e", e, rows * G);
    KT_TRY(apart(who, b, in));
    KT_TRY(apart(who, s, in));
    KT_TRY(apart(who, b, s));
    return launched(who, kt_launch_act8_save(dt, rows, cols, x, ldx, q, e, stream));
}

extern "C" kt_status kt_act8_restore(kt_dtype dt, int64_t rows, int64_t cols, const int8_t *q, const uint8_t *e, void *y,
                                     int64_t ldy, void *stream)
{
    const char *who = "kt_act8_restore";
    if (!is_type(dt)) return bad(who, "unknown element type");
    if (!sizes(rows, cols, ldy)) return bad(who, "rows >= 0, cols >= 1 and ld >= cols are needed");
    if (cols > MOST_ACT8_COLS) return unsupported(who, "more than 2^30 columns");
    if (rows == 0) return KT_OK;
    if (!q || !e || !y) return bad(who, "NULL q, e or y");
    KT_TRY(aligned(who, "y", y, size_of(dt)));
    KT_TRY(aligned(who, "q", q, 16));
    const int64_t G = kt_act8_groups(cols);
    const Block out = matrix("y", y, dt, rows, cols, ldy);
    KT_TRY(apart(who, out, flat("q", q, rows * G * KT_ACT8_GROUP)));
    KT_TRY(apart(who, out, flat("e", e, rows * G)));
    return launched(who, kt_launch_act8_restore(dt, rows, cols, q, e, y, ldy, stream));
}

static const int64_t MOST_WEIGHTS = 1 << 24;        // rows, columns: a step of the kernel has 31-bit offsets

static bool weight_grad_sizes(int64_t tokens, int64_t out, int64_t in)
{
    return tokens >= 0 && tokens <= (1ll << 40) && out >= 1 && in >= 1 && out <= MOST_WEIGHTS && in <= MOST_WEIGHTS;
}

extern "C" int64_t kt_act8_weight_grad_workspace(kt_dtype dt, int64_t tokens, int64_t out, int64_t in)
{
    return is_type(dt) && weight_grad_sizes(tokens, out, in) ? kt_weight_grad_ws(dt, tokens, out, in) : 0;
}

extern "C" kt_status kt_act8_weight_grad(kt_dtype dt, kt_dtype gdt, int64_t tokens, int64_t out, int64_t in, const void *dy,
                                         int64_t lddy, const int8_t *q, const uint8_t *e, void *dw, int64_t lddw, void *ws,
                                         int64_t ws_bytes, void *stream)
{
    const char *who = "kt_act8_weight_grad";
    if (!is_type(dt) || !is_type(gdt)) return bad(who, "unknown element type");
    if (!sizes(tokens, out, lddy) || !sizes(tokens, in, in) || !sizes(out, in, lddw)) return bad(who, "tokens >= 0, out and in >= 1 and ld >= columns are needed");
    if (!weight_grad_sizes(tokens, out, in)) return unsupported(who, "more than 2^40 tokens, or 2^24 rows or columns");
    if (!dw || (tokens && (!dy || !q || !e))) return bad(who, "NULL dy, q, e or dw");
    const int64_t need = kt_weight_grad_ws(dt, tokens, out, in);
    if (need && (!ws || ws_bytes < need)) return bad(who, "the workspace is smaller than kt_act8_weight_grad_workspace says");
    KT_TRY(aligned(who, "dy", dy, size_of(dt)));
    KT_TRY(aligned(who, "q", q, 16));
    KT_TRY(aligned(who, "dw", dw, size_of(gdt)));
    KT_TRY(aligned(who, "ws", ws, 16));
    const int64_t G = kt_act8_groups(in);
    const Block outs[] = {matrix("dw", dw, gdt, out, in, lddw), flat("ws", ws, need)};
    const Block ins[] = {matrix("dy", dy, dt, tokens, out, lddy), flat("q", q, tokens * G * KT_ACT8_GROUP), flat("e", e, tokens * G)};
    for (const Block &o : outs)
        for (const Block &i : ins) KT_TRY(apart(who, o, i));
    KT_TRY(apart(who, outs[1], outs[0]));
    return launched(who, kt_launch_weight_grad(dt, gdt, tokens, (int)out, (int)in, dy, lddy, q, e, dw, lddw, (float *)ws, stream));
}

// ---- attention -------------------------------------------------------------------

namespace {

const int64_t MOST_TOKENS = 1 << 30, MOST_HEADS = 1 << 16, MOST_STRIDE = 1ll << 40;

// A tensor of heads in memory; strides in bytes.
struct Spread {
    const char *name;
    const void *p;
    int64_t n[3], stride[3], dim;       // batch, tokens, heads
};
Spread spread(const char *name, const kt_heads *h, const kt_attention *a, int64_t tokens, int64_t heads)
{
    const int64_t s = size_of(a->dt);
    return Spread{name, h->data, {a->batch, tokens, heads}, {h->batch * s, h->token * s, h->head * s}, a->dim * s};
}
bool empty(const Spread &t) { return t.n[0] < 1 || t.n[1] < 1 || t.n[2] < 1; }
uintptr_t begin(const Spread &t) { return reinterpret_cast<uintptr_t>(t.p); }
// Bytes that the dimensions with strides below `ld` span; -1 where one of the others is no multiple of it.
int64_t extent(const Spread &t, int64_t ld)
{
    int64_t e = t.dim;
    for (int i = 0; i < 3; ++i) {
        if (t.n[i] < 2) continue;
        if (t.stride[i] < ld) e += (t.n[i] - 1) * t.stride[i];
        else if (t.stride[i] % ld) return -1;
    }
    return e;
}
// Whether two tensors provably share no byte: one ends before the other begins, or both are windows of one buffer that lie side
// by side within a token, a head or a sequence.
bool apart(const Spread &a, const Spread &b)
{
    if (empty(a) || empty(b)) return true;
    if (begin(a) + (uintptr_t)extent(a, INT64_MAX) <= begin(b) || begin(b) + (uintptr_t)extent(b, INT64_MAX) <= begin(a)) return true;
    for (int i = 0; i < 3; ++i) {
        const int64_t ld = a.stride[i];
        if (ld < 1) continue;
        const int64_t ea = extent(a, ld), eb = extent(b, ld);
        if (ea < 0 || eb < 0 || ea > ld || eb > ld) continue;
        const int64_t d = begin(b) >= begin(a) ? (int64_t)((begin(b) - begin(a)) % (uintptr_t)ld)
                                               : (ld - (int64_t)((begin(a) - begin(b)) % (uintptr_t)ld)) % ld;
        if (d >= ea && d + eb <= ld) return true;
    }
    return false;
}
// Whether no two elements of an output share an address: in order of their strides, each dimension steps over those below.
bool distinct(const Spread &t)
{
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (t.stride[order[j]] < t.stride[order[i]]) { const int x = order[i]; order[i] = order[j]; order[j] = x; }
    int64_t below = t.dim;
    for (int i : order) {
        if (t.n[i] < 2) continue;
        if (t.stride[i] < below) return false;
        below += (t.n[i] - 1) * t.stride[i];
    }
    return true;
}

// Whether a workgroup for every KT_ATTENTION_OWN tokens of every head makes fewer than 2^32 lanes: HIP launches no more.  batch * heads is
// at most 2^46.
bool launchable(int64_t batch, int64_t heads, int64_t tokens)
{
    const int64_t most = UINT32_MAX / KT_ATTENTION_BLOCK, blocks = (tokens + KT_ATTENTION_OWN - 1) / KT_ATTENTION_OWN;
    return blocks == 0 || batch * heads <= most / blocks;
}

// `bwd`: the backward pass also launches over the keys.
kt_status attention_sizes(const char *who, const kt_attention *a, bool bwd)
{
    if (!a) return bad(who, "NULL sizes");
    if (!is_type(a->dt)) return bad(who, "unknown element type");
    if (a->batch < 0 || a->nq < 0 || a->nk < 0 || a->heads < 1 || a->kv_heads < 1 || a->dim < 1) return bad(who, "negative sizes, or no heads or dim");
    if (a->heads % a->kv_heads) return bad(who, "kv_heads does not divide heads");
    if (!(a->scale > 0.0f) || std::isinf(a->scale)) return bad(who, "scale must be finite and > 0");
    if (a->dim > KT_ATTENTION_MAX_DIM) return unsupported(who, "dim over KT_ATTENTION_MAX_DIM");
    if (a->nq > MOST_TOKENS || a->nk > MOST_TOKENS || a->heads > MOST_HEADS || a->batch > MOST_TOKENS)
        return unsupported(who, "more than 2^30 queries, keys or sequences, or 2^16 heads");
    if (!launchable(a->batch, a->heads, a->nq) || (bwd && !launchable(a->batch, a->kv_heads, a->nk)))
        return unsupported(who, "2^24 workgroups or more, each 128 queries or keys of a head");
    return aligned(who, "k_lens", a->k_lens, 4);
}

kt_status heads_tensor(const char *who, const char *name, const kt_heads *h, const kt_attention *a, int64_t tokens, int64_t heads,
                       bool out)
{
    const bool none = a->batch == 0 || tokens == 0;
    if (!h || (!h->data && !none)) {
        kt_set_error("%s: NULL %s", who, name);
        return KT_EINVAL;
    }
    if (none) return KT_OK;
    if (h->batch < 0 || h->token < 0 || h->head < 0 || h->batch > MOST_STRIDE || h->token > MOST_STRIDE || h->head > MOST_STRIDE) {
        kt_set_error("%s: strides of %s are negative or over 2^40", who, name);
        return KT_EINVAL;
    }
    const int64_t room = INT64_MAX / 8;         // of a span in bytes
    if ((a->batch > 1 && h->batch > room / 4 / a->batch) || (tokens > 1 && h->token > room / 4 / tokens)) {
        kt_set_error("%s: %s spans more than 2^60 bytes", who, name);
        return KT_EINVAL;
    }
    const kt_status st = aligned(who, name, h->data, size_of(a->dt));
    if (st != KT_OK) return st;
    if (out && !distinct(spread(name, h, a, tokens, heads))) {
        kt_set_error("%s: elements of %s share addresses", who, name);
        return KT_EINVAL;
    }
    return KT_OK;
}

kt_status all_apart(const char *who, const Spread *outs, int no, const Spread *ins, int ni)
{
    for (int i = 0; i < no; ++i) {
        for (int j = 0; j < ni; ++j)
            if (!apart(outs[i], ins[j])) { kt_set_error("%s: %s overlaps %s", who, outs[i].name, ins[j].name); return KT_EINVAL; }
        for (int j = 0; j < i; ++j)
            if (!apart(outs[i], outs[j])) { kt_set_error("%s: %s overlaps %s", who, outs[i].name, outs[j].name); return KT_EINVAL; }
    }
    return KT_OK;
}

}  // namespace

extern "C" kt_status kt_attention_fwd(const kt_attention *a, const kt_heads *q, const kt_heads *k, const kt_heads *v,
                                      const kt_heads *o, float *lse, void *stream)
{
    const char *who = "kt_attention_fwd";
    KT_TRY(attention_sizes(who, a, false));
    KT_TRY(heads_tensor(who, "q", q, a, a->nq, a->heads, false));
    KT_TRY(heads_tensor(who, "k", k, a, a->nk, a->kv_heads, false));
    KT_TRY(heads_tensor(who, "v", v, a, a->nk, a->kv_heads, false));
    KT_TRY(heads_tensor(who, "o", o, a, a->nq, a->heads, true));
    KT_TRY(aligned(who, "lse", lse, 4));
    if (a->batch == 0 || a->nq == 0) return KT_OK;
    const int64_t stats = a->batch * a->heads * a->nq * 4;
    const Spread outs[] = {spread("o", o, a, a->nq, a->heads), Spread{"lse", lse, {lse ? 1 : 0, 1, 1}, {0, 0, 0}, stats}};
    const Spread ins[] = {spread("q", q, a, a->nq, a->heads), spread("k", k, a, a->nk, a->kv_heads), spread("v", v, a, a->nk, a->kv_heads),
                          Spread{"k_lens", a->k_lens, {a->k_lens ? 1 : 0, 1, 1}, {0, 0, 0}, a->batch * 4}};
    KT_TRY(all_apart(who, outs, 2, ins, 4));
    return launched(who, kt_launch_attention_fwd(a, q, k, v, o, lse, stream));
}

extern "C" int64_t kt_attention_bwd_workspace(const kt_attention *a)
{
    return attention_sizes("kt_attention_bwd_workspace", a, true) == KT_OK ? kt_attention_bwd_ws(a) : 0;
}

extern "C" kt_status kt_attention_bwd(const kt_attention *a, const kt_heads *d_o, const kt_heads *q, const kt_heads *k,
                                      const kt_heads *v, const kt_heads *o, const float *lse, const kt_heads *dq,
                                      const kt_heads *dk, const kt_heads *dv, void *ws, int64_t ws_bytes, void *stream)
{
    const char *who = "kt_attention_bwd";
    KT_TRY(attention_sizes(who, a, true));
    KT_TRY(heads_tensor(who, "d_o", d_o, a, a->nq, a->heads, false));
    KT_TRY(heads_tensor(who, "q", q, a, a->nq, a->heads, false));
    KT_TRY(heads_tensor(who, "k", k, a, a->nk, a->kv_heads, false));
    KT_TRY(heads_tensor(who, "v", v, a, a->nk, a->kv_heads, false));
    KT_TRY(heads_tensor(who, "o", o, a, a->nq, a->heads, false));
    KT_TRY(heads_tensor(who, "dq", dq, a, a->nq, a->heads, true));
    KT_TRY(heads_tensor(who, "dk", dk, a, a->nk, a->kv_heads, true));
    KT_TRY(heads_tensor(who, "dv", dv, a, a->nk, a->kv_heads, true));
    if (a->batch == 0) return KT_OK;
    const int64_t stats = a->batch * a->heads * a->nq * 4, need = kt_attention_bwd_ws(a);
    if (!lse && stats) return bad(who, "NULL lse");
    KT_TRY(aligned(who, "lse", lse, 4));
    if (need && (!ws || ws_bytes < need)) return bad(who, "the workspace is smaller than kt_attention_bwd_workspace says");
    KT_TRY(aligned(who, "ws", ws, 16));
    const Spread outs[] = {spread("dq", dq, a, a->nq, a->heads), spread("dk", dk, a, a->nk, a->kv_heads), spread("dv", dv, a, a->nk, a->kv_heads),
                           Spread{"ws", ws, {need ? 1 : 0, 1, 1}, {0, 0, 0}, need}};
    const Spread ins[] = {spread("d_o", d_o, a, a->nq, a->heads), spread("q", q, a, a->nq, a->heads), spread("k", k, a, a->nk, a->kv_heads),
                          spread("v", v, a, a->nk, a->kv_heads), spread("o", o, a, a->nq, a->heads),
                          Spread{"lse", lse, {stats ? 1 : 0, 1, 1}, {0, 0, 0}, stats},
                          Spread{"k_lens", a->k_lens, {a->k_lens ? 1 : 0, 1, 1}, {0, 0, 0}, a->batch * 4}};
    KT_TRY(all_apart(who, outs, 4, ins, 7));
    return launched(who, kt_launch_attention_bwd(a, d_o, q, k, v, o, lse, dq, dk, dv, (float *)ws, stream));
}
