// C entry points of the language-model operators (include/gpga.h): checks of arguments, scratch, dispatch.  Everything is
// refused before anything is launched.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "gpga_rows.hpp"

namespace {

gpga_status fail(gpga_ctx* c, gpga_status s, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(c->err, sizeof(c->err), fmt, ap);
    va_end(ap);
    return s;
}

gpga_status hip_fail(gpga_ctx* c, hipError_t e, const char* what) {
    return fail(c, e == hipErrorOutOfMemory ? GPGA_ENOMEM : GPGA_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// Makes the context's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool changed = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) == hipSuccess && prev != dev) changed = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        if (changed) (void)hipSetDevice(prev);
    }
};

// Scratch of one call; calls follow each other on the bound stream, so they share it.  What it outgrows stays until the context
// goes: a captured graph may hold its address.
gpga_status reserve(gpga_ctx* c, size_t bytes) {
    if (c->op_scratch_cap >= bytes) return GPGA_OK;
    constexpr size_t kLeast = (size_t)1 << 20;
    size_t want = c->op_scratch_cap + c->op_scratch_cap / 2;
    if (want < bytes) want = bytes;
    if (want < kLeast) want = kLeast;
    if (c->op_scratch && c->op_outgrown_count == kMaxOutgrown) return fail(c, GPGA_ENOMEM, "scratch has grown %d times", kMaxOutgrown);
    char* more = nullptr;
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&more), want);
    if (e == hipErrorOutOfMemory && want > bytes) {  // what is needed, where half as much again is not to be had
        (void)hipGetLastError();
        want = bytes;
        e = hipMalloc(reinterpret_cast<void**>(&more), want);
    }
    if (e != hipSuccess) {
        (void)hipGetLastError();  // reported here, not by the next call's launch
        return hip_fail(c, e, "hipMalloc(scratch)");
    }
    if (c->op_scratch) c->op_outgrown[c->op_outgrown_count++] = c->op_scratch;
    c->op_scratch = more;
    c->op_scratch_cap = want;
    return GPGA_OK;
}

int64_t elem_size(int32_t dtype) { return dtype == GPGA_F32 ? 4 : 2; }

constexpr int32_t kMaxTokens = 1 << 30;     // token numbers of a node are 32-bit
constexpr int32_t kMaxRow = 1 << 30;        // and so are column numbers
constexpr int64_t kMaxGroups = 0x7fffffff;  // rows of all nodes, and workgroups: numbered in 32 bits over all launches of a kernel

// An array of rows as a call sees it.
struct Array {
    const char* name;
    const void* p;
    bool out;
};

// The bytes of an array of rows of the call's shape, T > 0.
RowBytes row_bytes(const RowsShape& s, const void* p) {
    const int64_t size = elem_size(s.dtype);
    return {p, (int64_t)s.n * s.T, s.ld * size, s.D * size};
}

gpga_status check_ready(gpga_ctx* c) {
    if (!c->bound) return fail(c, GPGA_ESTATE, "buffers are not bound (gpga_bind)");
    return GPGA_OK;
}

// Shape and arrays common to all operators.  Outputs may take the place of an input exactly, and overlap nothing else; no input of a
// call that writes gradients lies in g.
gpga_status check_rows(gpga_ctx* c, const RowsShape& s, const Array* arrays, int count, bool writes_g = false) {
    if (s.dtype < GPGA_F32 || s.dtype > GPGA_F16) return fail(c, GPGA_EINVAL, "dtype %d is not a gpga_dtype", s.dtype);
    if (s.T < 0 || s.T > kMaxTokens) return fail(c, GPGA_EINVAL, "T = %d must be 0..%d", s.T, kMaxTokens);
    if (s.D < 1 || s.D > kMaxRow) return fail(c, GPGA_EINVAL, "a row has %d elements: it needs 1..%d", s.D, kMaxRow);
    if (s.ld < s.D) return fail(c, GPGA_EINVAL, "ld = %lld is smaller than the %d elements of a row", (long long)s.ld, s.D);
    const int64_t size = elem_size(s.dtype), rows = (int64_t)s.n * s.T;
    int64_t bytes = 0;
    if (rows > kMaxGroups) return fail(c, GPGA_EINVAL, "%lld rows: at most %lld", (long long)rows, (long long)kMaxGroups);
    if (__builtin_mul_overflow(rows, s.ld, &bytes) || __builtin_mul_overflow(bytes, size, &bytes) || bytes > (1ll << 56))
        return fail(c, GPGA_EINVAL, "%lld rows of ld = %lld are more than can be addressed", (long long)rows, (long long)s.ld);
    if (s.T == 0) return GPGA_OK;  // no row is touched
    const int64_t state = (int64_t)c->n * c->ld * (int64_t)sizeof(float);
    const struct {
        const char* name;
        const float* p;
    } held[4] = {{"x", c->x}, {"x_new", c->x_new}, {"m", c->m}, {"g", c->g}};
    for (int k = 0; k < count; ++k) {
        if (!arrays[k].p) continue;
        if (reinterpret_cast<uintptr_t>(arrays[k].p) & (uintptr_t)(size - 1)) return fail(c, GPGA_EINVAL, "%s is not aligned to its elements", arrays[k].name);
        for (const auto& h : held) {
            if (!arrays[k].out && !(writes_g && h.p == c->g)) continue;
            if (h.p && rows_meet_span(row_bytes(s, arrays[k].p), h.p, state))
                return fail(c, GPGA_EINVAL, "%s overlaps the bound array %s", arrays[k].name, h.name);
        }
        if (!arrays[k].out) continue;
        for (int j = 0; j < count; ++j) {
            if (j == k || !arrays[j].p || (arrays[j].p == arrays[k].p && !arrays[j].out)) continue;
            if (rows_meet(row_bytes(s, arrays[k].p), arrays[j].p))
                return fail(c, GPGA_EINVAL, "%s and %s overlap", arrays[k].name, arrays[j].name);
        }
    }
    return GPGA_OK;
}

// `floats` of fp32 that the call reads or writes beside its rows: they share no byte with an output or, written, with any array.
gpga_status check_floats(gpga_ctx* c, const RowsShape& s, const char* name, const float* p, int64_t floats, bool out, const Array* arrays, int count) {
    if (!p || !floats) return GPGA_OK;
    const int64_t bytes = floats * (int64_t)sizeof(float);
    for (int k = 0; k < count; ++k)
        if (s.T > 0 && arrays[k].p && (out || arrays[k].out) && rows_meet_span(row_bytes(s, arrays[k].p), p, bytes))
            return fail(c, GPGA_EINVAL, "%s and %s overlap", name, arrays[k].name);
    const int64_t state = (int64_t)c->n * c->ld * (int64_t)sizeof(float);
    const float* held[4] = {c->x, c->x_new, c->m, c->g};
    for (const float* h : held)
        if (h && (out || h == c->g) && rows_meet_span({h, 1, state, state}, p, bytes))
            return fail(c, GPGA_EINVAL, "%s overlaps a bound array", name);
    return GPGA_OK;
}

// `count` parameters of every node from column `off` on.
gpga_status check_columns(gpga_ctx* c, const char* name, int64_t off, int64_t count) {
    if (off < 0 || count > c->d || off > c->d - count)
        return fail(c, GPGA_EINVAL, "%s: columns %lld .. %lld + %lld are not within d = %lld", name, (long long)off, (long long)off, (long long)count,
                    (long long)c->d);
    return GPGA_OK;
}

// Tokens or labels, n * T of them, after check_rows: they share no byte with an output of the call.
gpga_status check_ints(gpga_ctx* c, const RowsShape& s, const char* name, const int32_t* p, const Array* arrays, int count, bool writes_g = false) {
    if (s.T > 0 && !p) return fail(c, GPGA_EINVAL, "%s must not be NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & 3u) return fail(c, GPGA_EINVAL, "%s is not 4-byte aligned", name);
    const int64_t bytes = (int64_t)s.n * s.T * (int64_t)sizeof(int32_t), state = (int64_t)c->n * c->ld * (int64_t)sizeof(float);
    for (int k = 0; k < count; ++k)
        if (s.T > 0 && arrays[k].p && arrays[k].out && rows_meet_span(row_bytes(s, arrays[k].p), p, bytes))
            return fail(c, GPGA_EINVAL, "%s and %s overlap", name, arrays[k].name);
    if (writes_g && rows_meet_span({c->g, 1, state, state}, p, bytes)) return fail(c, GPGA_EINVAL, "%s overlaps the bound array g", name);
    return GPGA_OK;
}

gpga_status check_table(gpga_ctx* c, int64_t table_off, int32_t V, int32_t D) {
    if (V < 1 || V > 0x7ffffff0) return fail(c, GPGA_EINVAL, "V = %d must be at least 1", V);
    if (D < 1) return fail(c, GPGA_EINVAL, "D = %d must be at least 1", D);
    return check_columns(c, "table", table_off, (int64_t)V * D);
}

// Dropout of iteration k in layer `layer`; p = 0 is none.
gpga_status make_drop(gpga_ctx* c, const RowsShape& s, float p, uint64_t seed, int32_t layer, DropArgs* out) {
    if (!(p >= 0.f && p < 1.f)) return fail(c, GPGA_EINVAL, "p = %g must be in [0, 1)", (double)p);
    if (layer < 0 || layer >= 1 << 24) return fail(c, GPGA_EINVAL, "layer = %d must be 0..%d", layer, (1 << 24) - 1);
    const uint32_t drop = (uint32_t)((double)p * 65536.0 + 0.5);
    if (drop >= 65536u) return fail(c, GPGA_EINVAL, "p = %.9g leaves nothing: it is kept to 16 bits", (double)p);
    const int64_t octs = ((int64_t)s.D + kOct - 1) / kOct;
    if (drop && (int64_t)s.T * octs > 0xffffffffll) return fail(c, GPGA_EINVAL, "T * ceil(D / 8) must be below 2^32 with dropout");
    out->k0 = (uint32_t)seed;
    out->k1 = (uint32_t)(seed >> 32);
    out->iter = (uint32_t)c->k;
    out->tag = TAG_DROPOUT | (uint32_t)layer << 8;
    out->drop = drop;
    out->factor = (float)(65536.0 / (65536.0 - (double)drop));
    return GPGA_OK;
}

#define GPGA_TRY(call)                        \
    do {                                      \
        const gpga_status s_ = (call);        \
        if (s_ != GPGA_OK) return s_;         \
    } while (0)

}  // namespace

extern "C" {

gpga_status gpga_embed(gpga_ctx* c, const int32_t* tokens, int32_t T, int64_t table_off, int32_t V, int32_t D, float scale, void* y, int64_t ld,
                       int32_t dtype) {
    if (!c) return GPGA_EINVAL;
    GPGA_TRY(check_ready(c));
    const RowsShape s = {c->n, T, D, ld, dtype};
    const Array arrays[] = {{"y_dev", y, true}};
    GPGA_TRY(check_table(c, table_off, V, D));
    GPGA_TRY(check_rows(c, s, arrays, 1));
    GPGA_TRY(check_ints(c, s, "tokens_dev", tokens, arrays, 1));
    if (!std::isfinite(scale)) return fail(c, GPGA_EINVAL, "scale must be finite");
    if (T == 0) return GPGA_OK;
    if (!y) return fail(c, GPGA_EINVAL, "y_dev must not be NULL");
    DeviceGuard guard(c->device);
    const hipError_t e = launch_embed(c, s, tokens, table_off, V, scale, y);
    return e == hipSuccess ? GPGA_OK : hip_fail(c, e, "embedding kernel launch");
}

gpga_status gpga_embed_grad(gpga_ctx* c, const int32_t* tokens, int32_t T, int64_t table_off, int32_t V, int32_t D, float scale, const void* dy,
                            int64_t ld, int32_t dtype, int32_t accumulate) {
    if (!c) return GPGA_EINVAL;
    GPGA_TRY(check_ready(c));
    const RowsShape s = {c->n, T, D, ld, dtype};
    const Array arrays[] = {{"dy_dev", dy, false}};
    GPGA_TRY(check_table(c, table_off, V, D));
    GPGA_TRY(check_rows(c, s, arrays, 1, true));
    GPGA_TRY(check_ints(c, s, "tokens_dev", tokens, arrays, 1, true));
    if (!std::isfinite(scale)) return fail(c, GPGA_EINVAL, "scale must be finite");
    if (accumulate != 0 && accumulate != 1) return fail(c, GPGA_EINVAL, "accumulate must be 0 or 1");
    if (T > 0 && !dy) return fail(c, GPGA_EINVAL, "dy_dev must not be NULL");
    if ((double)c->n * V * D / 1024 > 1e9) return fail(c, GPGA_EINVAL, "n * V * D must be below 10^12");
    DeviceGuard guard(c->device);
    GPGA_TRY(reserve(c, embed_grad_scratch(s)));
    const hipError_t e = launch_embed_grad(c, s, tokens, table_off, V, scale, dy, accumulate != 0, c->op_scratch);
    return e == hipSuccess ? GPGA_OK : hip_fail(c, e, "embedding gradient kernel launch");
}

gpga_status gpga_dropout(gpga_ctx* c, const void* x, const void* residual, int32_t T, int32_t D, int64_t ld, int32_t dtype, float p, uint64_t seed,
                         int32_t layer, void* y) {
    if (!c) return GPGA_EINVAL;
    GPGA_TRY(check_ready(c));
    const RowsShape s = {c->n, T, D, ld, dtype};
    const Array arrays[] = {{"x_dev", x, false}, {"residual_dev", residual, false}, {"y_dev", y, true}};
    DropArgs drop;
    GPGA_TRY(make_drop(c, s, p, seed, layer, &drop));
    GPGA_TRY(check_rows(c, s, arrays, 3));
    if (T == 0) return GPGA_OK;
    if (!x || !y) return fail(c, GPGA_EINVAL, "x_dev and y_dev must not be NULL");
    DeviceGuard guard(c->device);
    const hipError_t e = launch_dropout(c, s, drop, x, residual, y);
    return e == hipSuccess ? GPGA_OK : hip_fail(c, e, "dropout kernel launch");
}

gpga_status gpga_layer_norm(gpga_ctx* c, const void* x, const void* residual, int32_t T, int32_t D, int64_t ld, int32_t dtype, float p, uint64_t seed,
                            int32_t layer, int64_t gamma_off, int64_t beta_off, float eps, void* u, void* y, float* stats) {
    if (!c) return GPGA_EINVAL;
    GPGA_TRY(check_ready(c));
    const RowsShape s = {c->n, T, D, ld, dtype};
    const Array arrays[] = {{"x_dev", x, false}, {"residual_dev", residual, false}, {"u_dev", u, true}, {"y_dev", y, true}};
    GPGA_TRY(check_rows(c, s, arrays, 4));
    GPGA_TRY(check_columns(c, "gamma", gamma_off, D));
    GPGA_TRY(check_columns(c, "beta", beta_off, D));
    if (!(std::isfinite(eps) && eps >= 0.f)) return fail(c, GPGA_EINVAL, "eps must be finite and >= 0");
    if (reinterpret_cast<uintptr_t>(stats) & 3u) return fail(c, GPGA_EINVAL, "stats_dev is not 4-byte aligned");
    GPGA_TRY(check_floats(c, s, "stats_dev", stats, 2 * (int64_t)c->n * T, true, arrays, 4));
    DropArgs drop;
    GPGA_TRY(make_drop(c, s, p, seed, layer, &drop));
    if (T == 0) return GPGA_OK;
    if (!x || !y) return fail(c, GPGA_EINVAL, "x_dev and y_dev must not be NULL");
    DeviceGuard guard(c->device);
    const hipError_t e = launch_norm(c, s, drop, x, residual, gamma_off, beta_off, eps, u, y, stats);
    return e == hipSuccess ? GPGA_OK : hip_fail(c, e, "layer norm kernel launch");
}

gpga_status gpga_layer_norm_grad(gpga_ctx* c, const void* dy, const void* u, const float* stats, const void* more, int32_t T, int32_t D, int64_t ld,
                                 int32_t dtype, float p, uint64_t seed, int32_t layer, int64_t gamma_off, int64_t beta_off, void* du, void* dx,
                                 int32_t accumulate) {
    if (!c) return GPGA_EINVAL;
    GPGA_TRY(check_ready(c));
    const RowsShape s = {c->n, T, D, ld, dtype};
    const Array arrays[] = {{"dy_dev", dy, false}, {"u_dev", u, false}, {"more_dev", more, false}, {"du_dev", du, true}, {"dx_dev", dx, true}};
    GPGA_TRY(check_rows(c, s, arrays, 5, true));
    GPGA_TRY(check_columns(c, "gamma", gamma_off, D));
    GPGA_TRY(check_columns(c, "beta", beta_off, D));
    if (gamma_off < beta_off + D && beta_off < gamma_off + D) return fail(c, GPGA_EINVAL, "the columns of gamma and beta overlap");
    if (reinterpret_cast<uintptr_t>(stats) & 3u) return fail(c, GPGA_EINVAL, "stats_dev is not 4-byte aligned");
    if (accumulate != 0 && accumulate != 1) return fail(c, GPGA_EINVAL, "accumulate must be 0 or 1");
    GPGA_TRY(check_floats(c, s, "stats_dev", stats, 2 * (int64_t)c->n * T, false, arrays, 5));
    DropArgs drop;
    GPGA_TRY(make_drop(c, s, p, seed, layer, &drop));
    if (T > 0 && (!dy || !u || !stats || !du)) return fail(c, GPGA_EINVAL, "dy_dev, u_dev, stats_dev and du_dev must not be NULL");
    if (T > 0 && !dx && drop.drop) return fail(c, GPGA_EINVAL, "dx_dev may be NULL only when p == 0");
    if (T > 0 && dx && !drop.drop) return fail(c, GPGA_EINVAL, "dx_dev must be NULL when p == 0: du_dev is the gradient of x too");
    if ((int64_t)c->n * (((int64_t)D + 31) / 32) > kMaxGroups) return fail(c, GPGA_EINVAL, "n * D is too large");
    DeviceGuard guard(c->device);
    GPGA_TRY(reserve(c, norm_grad_scratch(s)));
    const hipError_t e = launch_norm_grad(c, s, drop, dy, u, stats, more, gamma_off, beta_off, du, dx, accumulate != 0, c->op_scratch);
    return e == hipSuccess ? GPGA_OK : hip_fail(c, e, "layer norm gradient kernel launch");
}

gpga_status gpga_token_loss(gpga_ctx* c, const void* logits, const int32_t* labels, int32_t T, int32_t V, int64_t ld, int32_t dtype, float grad_scale,
                            float* loss, void* dlogits) {
    if (!c) return GPGA_EINVAL;
    GPGA_TRY(check_ready(c));
    const RowsShape s = {c->n, T, V, ld, dtype};
    const Array arrays[] = {{"logits_dev", logits, false}, {"dlogits_dev", dlogits, true}};
    GPGA_TRY(check_rows(c, s, arrays, 2));
    GPGA_TRY(check_ints(c, s, "labels_dev", labels, arrays, 2));
    if (!std::isfinite(grad_scale)) return fail(c, GPGA_EINVAL, "grad_scale must be finite");
    if (!loss || (reinterpret_cast<uintptr_t>(loss) & 3u)) return fail(c, GPGA_EINVAL, "loss_dev must be a 4-byte aligned device pointer");
    if (T > 0 && !logits) return fail(c, GPGA_EINVAL, "logits_dev must not be NULL");
    GPGA_TRY(check_floats(c, s, "loss_dev", loss, c->n, true, arrays, 2));
    const int64_t losses = (int64_t)c->n * (int64_t)sizeof(float), ints = (int64_t)c->n * T * (int64_t)sizeof(int32_t);
    if (rows_meet_span({loss, 1, losses, losses}, labels, ints)) return fail(c, GPGA_EINVAL, "labels_dev and loss_dev overlap");
    DeviceGuard guard(c->device);
    GPGA_TRY(reserve(c, token_loss_scratch(s, c->num_cus)));
    const hipError_t e = launch_token_loss(c, s, logits, labels, grad_scale, loss, dlogits, c->op_scratch);
    return e == hipSuccess ? GPGA_OK : hip_fail(c, e, "token loss kernel launch");
}

}  // extern "C"
