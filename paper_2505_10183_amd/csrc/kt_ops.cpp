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
    return rows >= 0 && cols >= 1 && ld >= cols && ld <= most && (rows == 0 || ld <= most / rows);
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

static bool weight_grad_sizes(int64_t tokens, int64_t out, int64_t in)
{
    return tokens >= 0 && tokens <= (1ll << 40) && out >= 1 && in >= 1 && out <= MOST_ACT8_COLS && in <= MOST_ACT8_COLS && out * in <= (1ll << 46);
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
    if (!sizes(tokens, out, lddy) || !sizes(out, in, lddw)) return bad(who, "tokens >= 0, out and in >= 1 and ld >= columns are needed");
    if (!weight_grad_sizes(tokens, out, in)) return unsupported(who, "more than 2^40 tokens, 2^30 rows or columns, or 2^46 weights");
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
