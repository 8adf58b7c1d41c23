// C ABI of the SAMD library: argument validation (host only, before any HIP call),
// planning, and dispatch to the kernel launchers.
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <algorithm>
#include <string>
#include <vector>

#include "samd_internal.hpp"

namespace samd {

static thread_local std::string g_last_error;

void set_error(const std::string &msg) { g_last_error = msg; }

}  // namespace samd

using namespace samd;

namespace {

int fail(int status, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

int fail(int status, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_error(buf);
    return status;
}

int check_fmt(samd_fmt f, const char *name) {
    if (f.bits < 1 || f.bits > 8)
        return fail(SAMD_EINVAL, "%s.bits = %d is outside 1..8", name, f.bits);
    if (f.is_signed != 0 && f.is_signed != 1)
        return fail(SAMD_EINVAL, "%s.is_signed = %d must be 0 or 1", name, f.is_signed);
    return SAMD_OK;
}

bool aligned4(const void *p) { return ((uintptr_t)p & 3) == 0; }

int64_t max_abs(samd_fmt f) { return f.is_signed ? (int64_t)1 << (f.bits - 1) : ((int64_t)1 << f.bits) - 1; }

int check_conv2d_desc(const samd_conv2d_desc *d) {
    if (!d) return fail(SAMD_EINVAL, "descriptor is NULL");
    if (d->N < 1 || d->C < 1 || d->H < 1 || d->W < 1 || d->M < 1 || d->KH < 1 || d->KW < 1)
        return fail(SAMD_EINVAL, "shape N=%d C=%d H=%d W=%d M=%d KH=%d KW=%d must be positive", d->N, d->C,
                    d->H, d->W, d->M, d->KH, d->KW);
    if (d->stride_h < 1 || d->stride_w < 1 || d->pad_h < 0 || d->pad_w < 0)
        return fail(SAMD_EINVAL, "strides must be >= 1 and pads >= 0");
    if (d->pad_h >= d->KH || d->pad_w >= d->KW)
        return fail(SAMD_EINVAL, "padding must be smaller than the kernel");
    if (d->H + 2 * d->pad_h < d->KH || d->W + 2 * d->pad_w < d->KW)
        return fail(SAMD_EINVAL, "kernel larger than the padded input");
    return SAMD_OK;
}

// Exact int32 results: every output is a sum of C*KH*KW products of magnitude at most
// max|x| * max|w|.
int check_overflow(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf) {
    __int128 bound = (__int128)d->C * d->KH * d->KW * max_abs(xf) * max_abs(wf);
    if (bound >= ((__int128)1 << 31))
        return fail(SAMD_EOVERFLOW, "C*KH*KW*max|x|*max|w| = %lld does not fit int32", (long long)bound);
    return SAMD_OK;
}

}  // namespace

extern "C" {

const char *samd_status_str(int status) {
    switch (status) {
        case SAMD_OK: return "SAMD_OK";
        case SAMD_EINVAL: return "SAMD_EINVAL: invalid argument";
        case SAMD_EALIGN: return "SAMD_EALIGN: buffer not 4-byte aligned";
        case SAMD_EUNSUPPORTED: return "SAMD_EUNSUPPORTED: no exact lane geometry";
        case SAMD_EOVERFLOW: return "SAMD_EOVERFLOW: result may exceed int32";
        case SAMD_EHIP: return "SAMD_EHIP: HIP runtime error";
        case SAMD_ENOSPC: return "SAMD_ENOSPC: workspace too small";
        default: return "unknown SAMD status";
    }
}

const char *samd_last_error(void) { return g_last_error.c_str(); }

int64_t samd_row_words(int64_t len, samd_fmt f) {
    int st = check_fmt(f, "fmt");
    if (st) return st;
    if (len < 0) return fail(SAMD_EINVAL, "len = %lld is negative", (long long)len);
    return row_words(len, f.bits);
}

int samd_pack(const void *src, int64_t rows, int64_t len, samd_fmt f, uint32_t *dst, int32_t *oor_count,
              hipStream_t stream) {
    set_error("");
    int st = check_fmt(f, "fmt");
    if (st) return st;
    if (rows < 0 || len < 0) return fail(SAMD_EINVAL, "rows and len must be >= 0");
    if (rows == 0 || len == 0) return SAMD_OK;
    if (!src || !dst) return fail(SAMD_EINVAL, "src and dst must not be NULL");
    if (!aligned4(dst) || (oor_count && !aligned4(oor_count))) return fail(SAMD_EALIGN, "dst / oor_count not aligned");
    return launch_pack(src, rows, len, f.bits, f.is_signed, dst, oor_count, stream);
}

int samd_unpack(const uint32_t *src, int64_t rows, int64_t len, samd_fmt f, void *dst, hipStream_t stream) {
    set_error("");
    int st = check_fmt(f, "fmt");
    if (st) return st;
    if (rows < 0 || len < 0) return fail(SAMD_EINVAL, "rows and len must be >= 0");
    if (rows == 0 || len == 0) return SAMD_OK;
    if (!src || !dst) return fail(SAMD_EINVAL, "src and dst must not be NULL");
    if (!aligned4(src)) return fail(SAMD_EALIGN, "src not aligned");
    return launch_unpack(src, rows, len, f.bits, f.is_signed, dst, stream);
}

}  // extern "C"

namespace {

// Checks shared by samd_conv1d and its plan query; plans into g.
int conv1d_checks(int64_t n, samd_fmt xf, const int32_t *taps, int32_t K, samd_fmt kf, Conv1dGeom &g) {
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(kf, "kf");
    if (st) return st;
    if (xf.is_signed || kf.is_signed) return fail(SAMD_EINVAL, "samd_conv1d takes unsigned operands");
    if (!taps) return fail(SAMD_EINVAL, "taps must not be NULL");
    if (K < 1 || K > 16) return fail(SAMD_EINVAL, "K = %d is outside 1..16", K);
    if (n < K) return fail(SAMD_EINVAL, "n = %lld is shorter than the kernel", (long long)n);
    if (row_words(n, xf.bits) > INT32_MAX || n > ((int64_t)1 << 40))
        return fail(SAMD_EINVAL, "n = %lld too large", (long long)n);
    for (int t = 0; t < K; ++t)
        if (taps[t] < 0 || taps[t] > (1 << kf.bits) - 1)
            return fail(SAMD_EINVAL, "tap %d = %d outside the %d-bit unsigned range", t, taps[t], kf.bits);
    __int128 bound = (__int128)K * (((int64_t)1 << xf.bits) - 1) * (((int64_t)1 << kf.bits) - 1);
    if (bound >= ((__int128)1 << 31)) return fail(SAMD_EOVERFLOW, "K*max|x|*max|k| does not fit int32");
    std::string err;
    st = plan_conv1d(n, xf, taps, K, kf, g, err);
    if (st) return fail(st, "%s", err.c_str());
    return SAMD_OK;
}

}  // namespace

extern "C" {

int samd_conv1d(const uint32_t *x, int64_t n, samd_fmt xf, const int32_t *taps, int32_t K, samd_fmt kf,
                int32_t *y, hipStream_t stream) {
    set_error("");
    Conv1dGeom g;
    int st = conv1d_checks(n, xf, taps, K, kf, g);
    if (st) return st;
    if (!x || !y) return fail(SAMD_EINVAL, "x and y must not be NULL");
    if (!aligned4(x) || !aligned4(y)) return fail(SAMD_EALIGN, "x / y not aligned");
    return launch_conv1d(x, g, y, stream);
}

int samd_conv1d_plan_query(int64_t n, samd_fmt xf, const int32_t *taps, int32_t K, samd_fmt kf,
                           samd_conv1d_plan *out) {
    set_error("");
    Conv1dGeom g;
    int st = conv1d_checks(n, xf, taps, K, kf, g);
    if (st) return st;
    if (!out) return fail(SAMD_EINVAL, "out must not be NULL");
    *out = samd_conv1d_plan{};
    out->lane_bits = g.L;
    out->lanes = g.I;
    out->groups = g.ngroups;
    out->extra = g.extra;
    out->out_lanes = g.nl;
    for (int q = 0; q < g.ngroups; ++q) {
        out->tap0[q] = g.g_tap0[q];
        out->ntaps[q] = g.g_ntaps[q];
    }
    return SAMD_OK;
}

}  // extern "C"

namespace {

void fill_plan(const Conv2dGeom &g, samd_conv2d_plan *out) {
    *out = samd_conv2d_plan{};
    out->lane_bits = g.L;
    out->lanes = g.I;
    out->taps_max = g.Kmax;
    out->words_per_row = g.nq;
    out->flush_channels = g.G;
    out->out_lanes = g.nl;
    out->tap_words = g.ntw;
    for (int t = 0; t < g.ntw; ++t) {
        out->phase[t] = g.tw_phase[t];
        out->tap0[t] = g.tw_tap0[t];
        out->ntaps[t] = g.tw_ntaps[t];
    }
    out->rows_per_block = g.rows_blk;
    out->mblock = g.mblk;
    out->split_waves = g.ks;
    out->chunk_channels = g.chk;
    out->x_offset = g.xoff;
    out->col_segments = g.ncs;
    out->segment_columns = g.cw;
    out->macs_per_mad = g.macs_per_mad;
    out->rows_per_thread = g.rh;
    out->shared_rows = g.rows_path;
    out->model_cost = g.cost;
    out->layout_spaced = g.layout_spaced;
    out->spacer_msb = g.spacer;
}

}  // namespace

extern "C" {

int samd_conv2d_plan_query(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, samd_conv2d_plan *out) {
    set_error("");
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (!out) return fail(SAMD_EINVAL, "out must not be NULL");
    Conv2dGeom g;
    std::string err;
    st = plan_conv2d(*d, xf, wf, g, err);
    if (st) return fail(st, "%s", err.c_str());
    fill_plan(g, out);
    return SAMD_OK;
}

int samd_conv2d_form_query(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t layout_spaced,
                           samd_conv2d_form *out) {
    set_error("");
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (!out) return fail(SAMD_EINVAL, "out must not be NULL");
    Conv2dGeom g;
    std::string err;
    st = plan_conv2d(*d, xf, wf, g, err, layout_spaced ? 1 : 0);
    if (st) return fail(st, "%s", err.c_str());
    *out = samd_conv2d_form{conv2d_kernel_rows(g), g.two, g.period, g.result_signed, g.odd_mask};
    return SAMD_OK;
}

int samd_conv2d_workspace(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, size_t *bytes) {
    set_error("");
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (!bytes) return fail(SAMD_EINVAL, "bytes must not be NULL");
    Conv2dGeom g;
    std::string err;
    st = plan_conv2d(*d, xf, wf, g, err);
    if (st) return fail(st, "%s", err.c_str());
    *bytes = conv2d_workspace_bytes(g);
    return SAMD_OK;
}

}  // extern "C"

namespace {

// Validation and planning shared by the SAMD conv2d entry points.
int conv2d_setup(samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, const void *ws, size_t ws_bytes,
                 Conv2dGeom &g) {
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (!ws) return fail(SAMD_EINVAL, "ws must not be NULL");
    if (((uintptr_t)ws & 255) != 0) return fail(SAMD_EALIGN, "workspace not 256-byte aligned");
    std::string err;
    st = plan_conv2d(*d, xf, wf, g, err);
    if (st) return fail(st, "%s", err.c_str());
    size_t need = conv2d_workspace_bytes(g);
    if (ws_bytes < need) return fail(SAMD_ENOSPC, "workspace %zu bytes < %zu needed", ws_bytes, need);
    return SAMD_OK;
}

}  // namespace

extern "C" {

int samd_conv2d_prepare(const uint32_t *w, samd_fmt wf, const samd_conv2d_desc *d, samd_fmt xf, void *ws,
                        size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = conv2d_setup(xf, wf, d, ws, ws_bytes, g);
    if (st) return st;
    if (!w) return fail(SAMD_EINVAL, "w must not be NULL");
    if (!aligned4(w)) return fail(SAMD_EALIGN, "w not aligned");
    return launch_conv2d_prepare(w, g, ws, stream);
}

int samd_conv2d_prepared(const uint32_t *x, samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, int32_t *y,
                         const void *ws, size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = conv2d_setup(xf, wf, d, ws, ws_bytes, g);
    if (st) return st;
    if (!x || !y) return fail(SAMD_EINVAL, "x and y must not be NULL");
    if (!aligned4(x) || !aligned4(y)) return fail(SAMD_EALIGN, "x / y not aligned");
    return launch_conv2d_samd(x, g, y, ws, stream);
}

int samd_conv2d_stage(const uint32_t *x, samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, void *ws,
                      size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = conv2d_setup(xf, wf, d, ws, ws_bytes, g);
    if (st) return st;
    if (!x) return fail(SAMD_EINVAL, "x must not be NULL");
    if (!aligned4(x)) return fail(SAMD_EALIGN, "x not aligned");
    return launch_conv2d_spread(x, g, ws, stream);
}

int samd_relu_requant_stage(const int32_t *acc, const int32_t *dev_max, samd_fmt xf, samd_fmt wf,
                            const samd_conv2d_desc *d, void *ws, size_t ws_bytes, int32_t *dev_shift,
                            hipStream_t stream) {
    set_error("");
    if (xf.is_signed) return fail(SAMD_EINVAL, "requantised activations are unsigned");
    Conv2dGeom g;
    int st = conv2d_setup(xf, wf, d, ws, ws_bytes, g);
    if (st) return st;
    if (!acc || !dev_max) return fail(SAMD_EINVAL, "acc and dev_max must not be NULL");
    if (!aligned4(acc) || !aligned4(dev_max) || (dev_shift && !aligned4(dev_shift)))
        return fail(SAMD_EALIGN, "acc / dev_max / dev_shift not aligned");
    return launch_relu_requant_stage(acc, dev_max, g, ws, dev_shift, stream);
}

int samd_conv2d_accumulate(samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, int32_t *y, const void *ws,
                           size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = conv2d_setup(xf, wf, d, ws, ws_bytes, g);
    if (st) return st;
    if (!y) return fail(SAMD_EINVAL, "y must not be NULL");
    if (!aligned4(y)) return fail(SAMD_EALIGN, "y not aligned");
    return launch_conv2d_multiply(g, y, ws, stream);
}

int samd_conv2d(const uint32_t *x, samd_fmt xf, const uint32_t *w, samd_fmt wf, const samd_conv2d_desc *d,
                int32_t *y, void *ws, size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = conv2d_setup(xf, wf, d, ws, ws_bytes, g);
    if (st) return st;
    if (!x || !w || !y) return fail(SAMD_EINVAL, "x, w and y must not be NULL");
    if (!aligned4(x) || !aligned4(w) || !aligned4(y)) return fail(SAMD_EALIGN, "x / w / y not aligned");
    st = launch_conv2d_prepare(w, g, ws, stream);
    if (st) return st;
    return launch_conv2d_samd(x, g, y, ws, stream);
}

}  // extern "C"

namespace {

// Validation and planning shared by the permanent-spacer entry points (ws may be NULL
// where no workspace is used).
int spaced_setup(samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, Conv2dGeom &g) {
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    std::string err;
    st = plan_conv2d(*d, xf, wf, g, err, 1);
    if (st) return fail(st, "%s", err.c_str());
    return SAMD_OK;
}

int spaced_ws(const Conv2dGeom &g, const void *ws, size_t ws_bytes) {
    if (!ws) return fail(SAMD_EINVAL, "ws must not be NULL");
    if (((uintptr_t)ws & 255) != 0) return fail(SAMD_EALIGN, "workspace not 256-byte aligned");
    const size_t need = conv2d_xs_offset(g);
    if (ws_bytes < need) return fail(SAMD_ENOSPC, "workspace %zu bytes < %zu needed", ws_bytes, need);
    return SAMD_OK;
}

}  // namespace

extern "C" {

int samd_conv2d_spaced_plan_query(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, samd_conv2d_plan *out) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (st) return st;
    if (!out) return fail(SAMD_EINVAL, "out must not be NULL");
    fill_plan(g, out);
    return SAMD_OK;
}

int samd_conv2d_spaced_layout(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, samd_spaced_layout *out) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (st) return st;
    if (!out) return fail(SAMD_EINVAL, "out must not be NULL");
    *out = samd_spaced_layout{};
    out->lane_bits = g.L;
    out->lanes = g.I;
    out->words_per_row = g.nq;
    out->tap_words = g.ntw;
    out->padded_rows = g.Hp;
    out->x_offset = g.xoff;
    out->spacer_msb = g.spacer;
    out->words = g.spread_words + (int64_t)g.Hp * g.ntw * g.nq;
    return SAMD_OK;
}

int samd_conv2d_spaced_workspace(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, size_t *bytes) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (st) return st;
    if (!bytes) return fail(SAMD_EINVAL, "bytes must not be NULL");
    *bytes = conv2d_xs_offset(g);
    return SAMD_OK;
}

int samd_conv2d_spaced_prepare(const uint32_t *w, samd_fmt wf, const samd_conv2d_desc *d, samd_fmt xf, void *ws,
                               size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (!st) st = spaced_ws(g, ws, ws_bytes);
    if (st) return st;
    if (!w) return fail(SAMD_EINVAL, "w must not be NULL");
    if (!aligned4(w)) return fail(SAMD_EALIGN, "w not aligned");
    return launch_conv2d_prepare(w, g, ws, stream);
}

int samd_conv2d_spaced_pack(const void *src, samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, uint32_t *dst,
                            hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (st) return st;
    if (!src || !dst) return fail(SAMD_EINVAL, "src and dst must not be NULL");
    if (!aligned4(dst)) return fail(SAMD_EALIGN, "dst not aligned");
    return launch_conv2d_spread_bytes(src, g, (int32_t *)dst, stream);
}

int samd_conv2d_spaced_from_packed(const uint32_t *x, samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d,
                                   uint32_t *dst, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (st) return st;
    if (!x || !dst) return fail(SAMD_EINVAL, "x and dst must not be NULL");
    if (!aligned4(x) || !aligned4(dst)) return fail(SAMD_EALIGN, "x / dst not aligned");
    return launch_conv2d_spread(x, g, nullptr, stream, (int32_t *)dst);
}

int samd_conv2d_spaced(const uint32_t *xs, samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, int32_t *y,
                       const void *ws, size_t ws_bytes, hipStream_t stream) {
    set_error("");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (!st) st = spaced_ws(g, ws, ws_bytes);
    if (st) return st;
    if (!xs || !y) return fail(SAMD_EINVAL, "xs and y must not be NULL");
    if (!aligned4(xs) || !aligned4(y)) return fail(SAMD_EALIGN, "xs / y not aligned");
    return launch_conv2d_multiply(g, y, ws, stream, (const int32_t *)xs);
}

int samd_relu_requant_spaced(const int32_t *acc, const int32_t *dev_max, samd_fmt xf, samd_fmt wf,
                             const samd_conv2d_desc *d, uint32_t *dst, int32_t *dev_shift, hipStream_t stream) {
    set_error("");
    if (xf.is_signed) return fail(SAMD_EINVAL, "requantised activations are unsigned");
    Conv2dGeom g;
    int st = spaced_setup(xf, wf, d, g);
    if (st) return st;
    if (!acc || !dev_max || !dst) return fail(SAMD_EINVAL, "acc, dev_max and dst must not be NULL");
    if (!aligned4(acc) || !aligned4(dev_max) || !aligned4(dst) || (dev_shift && !aligned4(dev_shift)))
        return fail(SAMD_EALIGN, "acc / dev_max / dst / dev_shift not aligned");
    return launch_relu_requant_stage(acc, dev_max, g, nullptr, dev_shift, stream, (int32_t *)dst);
}

int samd_conv2d_noalloc(const uint32_t *x, samd_fmt xf, const uint32_t *w, samd_fmt wf, const samd_conv2d_desc *d,
                        int32_t *y, hipStream_t stream) {
    set_error("");
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (!x || !w || !y) return fail(SAMD_EINVAL, "x, w and y must not be NULL");
    if (!aligned4(x) || !aligned4(w) || !aligned4(y)) return fail(SAMD_EALIGN, "x / w / y not aligned");
    Conv2dGeom g;
    std::string err;
    st = plan_conv2d_scratch(*d, xf, wf, g, err);
    if (st) return fail(st, "%s", err.c_str());
    const size_t need = conv2d_workspace_bytes(g);
    if (need > (size_t)SAMD_NOALLOC_SCRATCH_BYTES)
        return fail(SAMD_ENOSPC, "the layer needs a %zu-byte workspace; the scratch array holds %zu bytes", need,
                    (size_t)SAMD_NOALLOC_SCRATCH_BYTES);
    return launch_conv2d_noalloc(x, w, g, y, stream);
}

namespace {

// The 8-bit baseline takes signed activations, or unsigned ones of up to 8 bits, and
// signed weights (8-bit unsigned weights do not fit int8).
int check_int8_formats(samd_fmt xf, samd_fmt wf) {
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (st) return st;
    if (!wf.is_signed && wf.bits == 8) return fail(SAMD_EINVAL, "8-bit unsigned weights do not fit int8");
    return SAMD_OK;
}

}  // namespace

int samd_conv2d_int8_workspace(const samd_conv2d_desc *d, samd_fmt xf, size_t *bytes) {
    set_error("");
    int st = check_fmt(xf, "xf");
    if (!st) st = check_conv2d_desc(d);
    if (st) return st;
    if (!bytes) return fail(SAMD_EINVAL, "bytes must not be NULL");
    *bytes = conv2d_i8_workspace_bytes(*d, xf);
    return SAMD_OK;
}

}  // extern "C"

namespace {

int int8_setup(samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, const void *ws, size_t ws_bytes) {
    int st = check_int8_formats(xf, wf);
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    // the kernel addresses the activations and 128 filters' reordered weights with
    // 32-bit byte offsets
    const int64_t cp = (d->C + 127) / 128 * 128;
    if ((int64_t)d->N * d->H * d->W * d->C >= ((int64_t)1 << 31) ||
        (int64_t)128 * d->KH * d->KW * cp >= ((int64_t)1 << 31))
        return fail(SAMD_EUNSUPPORTED, "the activations or 128 filters exceed 2 GiB");
    if (!ws) return fail(SAMD_EINVAL, "ws must not be NULL");
    if (((uintptr_t)ws & 255) != 0) return fail(SAMD_EALIGN, "workspace not 256-byte aligned");
    size_t need = conv2d_i8_workspace_bytes(*d, xf);
    if (ws_bytes < need) return fail(SAMD_ENOSPC, "workspace %zu bytes < %zu needed", ws_bytes, need);
    return SAMD_OK;
}

}  // namespace

extern "C" {

int samd_conv2d_int8_plan_query(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, samd_conv2d_int8_plan *out) {
    set_error("");
    int st = check_int8_formats(xf, wf);
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (!out) return fail(SAMD_EINVAL, "out must not be NULL");
    return conv2d_i8_tiles(*d, xf, *out);
}

int samd_conv2d_int8_candidates(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t max_count,
                                samd_conv2d_int8_plan *out, int32_t *count) {
    set_error("");
    int st = check_int8_formats(xf, wf);
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (max_count < 1 || max_count > SAMD_MAX_CANDIDATES)
        return fail(SAMD_EINVAL, "candidate count %d is outside 1..%d", max_count, SAMD_MAX_CANDIDATES);
    if (!out || !count) return fail(SAMD_EINVAL, "out and count must not be NULL");
    std::vector<samd_conv2d_int8_plan> cands;
    conv2d_i8_candidates(*d, xf, cands);
    const int n = std::min<int>(max_count, (int)cands.size());
    for (int i = 0; i < n; ++i) out[i] = cands[i];
    *count = n;
    return SAMD_OK;
}

int samd_conv2d_int8_use_plan(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, const samd_conv2d_int8_plan *plan) {
    set_error("");
    int st = check_int8_formats(xf, wf);
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    st = conv2d_i8_use_plan(*d, xf, plan);
    if (st) return fail(st, "%s", samd_last_error());
    return SAMD_OK;
}

int samd_conv2d_int8_prepare(const int8_t *w, samd_fmt wf, const samd_conv2d_desc *d, samd_fmt xf, void *ws,
                             size_t ws_bytes, hipStream_t stream) {
    set_error("");
    int st = int8_setup(xf, wf, d, ws, ws_bytes);
    if (st) return st;
    if (!w) return fail(SAMD_EINVAL, "w must not be NULL");
    return launch_conv2d_i8_prepare(w, xf, *d, ws, stream);
}

int samd_conv2d_int8_prepared(const void *x, samd_fmt xf, samd_fmt wf, const samd_conv2d_desc *d, int32_t *y,
                              const void *ws, size_t ws_bytes, hipStream_t stream) {
    set_error("");
    int st = int8_setup(xf, wf, d, ws, ws_bytes);
    if (st) return st;
    if (!x || !y) return fail(SAMD_EINVAL, "x and y must not be NULL");
    if (!aligned4(y)) return fail(SAMD_EALIGN, "y not aligned");
    return launch_conv2d_i8(x, xf, *d, y, ws, stream);
}

int samd_conv2d_int8(const void *x, samd_fmt xf, const int8_t *w, samd_fmt wf, const samd_conv2d_desc *d,
                     int32_t *y, void *ws, size_t ws_bytes, hipStream_t stream) {
    set_error("");
    int st = int8_setup(xf, wf, d, ws, ws_bytes);
    if (st) return st;
    if (!x || !w || !y) return fail(SAMD_EINVAL, "x, w and y must not be NULL");
    if (!aligned4(y)) return fail(SAMD_EALIGN, "y not aligned");
    st = launch_conv2d_i8_prepare(w, xf, *d, ws, stream);
    if (st) return st;
    return launch_conv2d_i8(x, xf, *d, y, ws, stream);
}

int samd_max_i32(const int32_t *src, int64_t n, int32_t *dev_max, hipStream_t stream) {
    set_error("");
    if (n < 1) return fail(SAMD_EINVAL, "n must be >= 1");
    if (!src || !dev_max) return fail(SAMD_EINVAL, "src and dev_max must not be NULL");
    if (!aligned4(src) || !aligned4(dev_max)) return fail(SAMD_EALIGN, "src / dev_max not aligned");
    return launch_max_i32(src, n, dev_max, stream);
}

int samd_lanewise(int op, const uint32_t *a, const uint32_t *b, int64_t nwords, samd_fmt f, uint32_t *dst,
                  hipStream_t stream) {
    set_error("");
    int st = check_fmt(f, "f");
    if (st) return st;
    if (op != SAMD_LANE_ADD && op != SAMD_LANE_SUB && op != SAMD_LANE_MUL)
        return fail(SAMD_EINVAL, "op %d is not SAMD_LANE_ADD, SAMD_LANE_SUB or SAMD_LANE_MUL", op);
    if (nwords < 0) return fail(SAMD_EINVAL, "nwords must be >= 0");
    if (nwords == 0) return SAMD_OK;
    if (!a || !b || !dst) return fail(SAMD_EINVAL, "a, b and dst must not be NULL");
    if (((uintptr_t)a & 15) || ((uintptr_t)b & 15) || ((uintptr_t)dst & 15))
        return fail(SAMD_EALIGN, "a, b and dst must be 16-byte aligned");
    return launch_lanewise(op, a, b, nwords, f.bits, 0, dst, stream);
}

int samd_scale(const uint32_t *a, int64_t nwords, samd_fmt f, int32_t scalar, uint32_t *dst, hipStream_t stream) {
    set_error("");
    int st = check_fmt(f, "f");
    if (st) return st;
    if (nwords < 0) return fail(SAMD_EINVAL, "nwords must be >= 0");
    if (nwords == 0) return SAMD_OK;
    if (!a || !dst) return fail(SAMD_EINVAL, "a and dst must not be NULL");
    if (((uintptr_t)a & 15) || ((uintptr_t)dst & 15)) return fail(SAMD_EALIGN, "a and dst must be 16-byte aligned");
    const uint32_t s = (uint32_t)scalar & ((1u << f.bits) - 1);   // the scalar's b-bit pattern
    return launch_lanewise(SAMD_LANE_SCALE, a, a, nwords, f.bits, s, dst, stream);
}

int samd_relu_requant_pack(const int32_t *acc, int64_t rows, int64_t len, const int32_t *dev_max, samd_fmt out,
                           uint32_t *dst, int32_t *dev_shift, hipStream_t stream) {
    set_error("");
    int st = check_fmt(out, "out");
    if (st) return st;
    if (out.is_signed) return fail(SAMD_EINVAL, "requantised activations are unsigned");
    if (rows < 0 || len < 0) return fail(SAMD_EINVAL, "rows and len must be >= 0");
    if (!acc || !dev_max || !dst) return fail(SAMD_EINVAL, "acc, dev_max and dst must not be NULL");
    if (!aligned4(acc) || !aligned4(dst) || !aligned4(dev_max) || (dev_shift && !aligned4(dev_shift)))
        return fail(SAMD_EALIGN, "buffer not aligned");
    if (rows == 0 || len == 0) return SAMD_OK;
    return launch_relu_requant_pack(acc, rows, len, dev_max, out.bits, dst, dev_shift, stream);
}

int samd_relu_requant_nhwc_u8(const int32_t *acc, int32_t N, int32_t C, int32_t H, int32_t W,
                              const int32_t *dev_max, samd_fmt out, uint8_t *dst, hipStream_t stream) {
    set_error("");
    int st = check_fmt(out, "out");
    if (st) return st;
    if (out.is_signed) return fail(SAMD_EINVAL, "requantised activations are unsigned");
    if (N < 1 || C < 1 || H < 1 || W < 1) return fail(SAMD_EINVAL, "shape must be positive");
    if (!acc || !dev_max || !dst) return fail(SAMD_EINVAL, "acc, dev_max and dst must not be NULL");
    if (!aligned4(acc) || !aligned4(dev_max)) return fail(SAMD_EALIGN, "buffer not aligned");
    return launch_relu_requant_nhwc_u8(acc, N, C, H, W, dev_max, out.bits, dst, stream);
}

// ---------------------------------------------------------------------------------------
// Autotuning: candidate plans ranked by the model, timed on the device.

}  // extern "C"

namespace {

// Shared validation of the candidate queries and the tuner.
int check_tune_args(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t count) {
    int st = check_fmt(xf, "xf");
    if (!st) st = check_fmt(wf, "wf");
    if (!st) st = check_conv2d_desc(d);
    if (!st) st = check_overflow(d, xf, wf);
    if (st) return st;
    if (count < 1 || count > SAMD_MAX_CANDIDATES)
        return fail(SAMD_EINVAL, "candidate count %d is outside 1..%d", count, SAMD_MAX_CANDIDATES);
    return SAMD_OK;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Bytes of one output tensor (the tuner's second output) and of its mismatch counter.
size_t tune_extra_bytes(const samd_conv2d_desc &d, const Conv2dGeom &g) {
    return round256((size_t)d.N * d.M * g.Ho * g.Wo * 4) + 256;
}

}  // namespace

extern "C" {

int samd_conv2d_candidates(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t max_count,
                           samd_conv2d_plan *out, int32_t *count) {
    set_error("");
    int st = check_tune_args(d, xf, wf, max_count);
    if (st) return st;
    if (!out || !count) return fail(SAMD_EINVAL, "out and count must not be NULL");
    std::vector<Conv2dGeom> cands;
    std::string err;
    st = conv2d_candidates(*d, xf, wf, max_count, cands, err);
    if (st) return fail(st, "%s", err.c_str());
    for (size_t i = 0; i < cands.size(); ++i) fill_plan(cands[i], out + i);
    *count = (int32_t)cands.size();
    return SAMD_OK;
}

}  // extern "C"

namespace {

int tune_workspace_impl(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t candidates, size_t *bytes,
                        int spaced) {
    set_error("");
    int st = check_tune_args(d, xf, wf, candidates);
    if (st) return st;
    if (!bytes) return fail(SAMD_EINVAL, "bytes must not be NULL");
    std::vector<Conv2dGeom> cands;
    std::string err;
    st = conv2d_candidates(*d, xf, wf, candidates, cands, err, spaced);
    if (st) return fail(st, "%s", err.c_str());
    size_t most = 0;
    for (const Conv2dGeom &c : cands) most = std::max(most, conv2d_workspace_bytes(c));
    *bytes = most + tune_extra_bytes(*d, cands[0]);
    return SAMD_OK;
}

}  // namespace

extern "C" {

int samd_conv2d_tune_workspace(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t candidates,
                               size_t *bytes) {
    return tune_workspace_impl(d, xf, wf, candidates, bytes, 0);
}

int samd_conv2d_spaced_tune_workspace(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, int32_t candidates,
                                      size_t *bytes) {
    return tune_workspace_impl(d, xf, wf, candidates, bytes, 1);
}

}  // extern "C"

namespace {

// The tuner of both layouts.  Packed layout: each timed run is stage + accumulate.
// Permanent-spacer layout: each candidate's operand words are written once (untimed) and
// the timed run is the multiply alone - the spaced convolution.
int tune_impl(const uint32_t *x, samd_fmt xf, const uint32_t *w, samd_fmt wf, const samd_conv2d_desc *d,
              int32_t *y, void *ws, size_t ws_bytes, int32_t candidates, int32_t reps, samd_conv2d_plan *chosen,
              hipStream_t stream, int spaced) {
    set_error("");
    int st = check_tune_args(d, xf, wf, candidates);
    if (st) return st;
    if (reps < 1 || reps > 1000) return fail(SAMD_EINVAL, "reps = %d is outside 1..1000", reps);
    if (!x || !w || !y || !ws) return fail(SAMD_EINVAL, "x, w, y and ws must not be NULL");
    if (!aligned4(x) || !aligned4(w) || !aligned4(y)) return fail(SAMD_EALIGN, "x / w / y not aligned");
    if (((uintptr_t)ws & 255) != 0) return fail(SAMD_EALIGN, "workspace not 256-byte aligned");
    std::vector<Conv2dGeom> cands;
    std::string err;
    st = conv2d_candidates(*d, xf, wf, candidates, cands, err, spaced);
    if (st) return fail(st, "%s", err.c_str());
    // the candidates whose workspace fits next to the second output and its counter
    const size_t extra = tune_extra_bytes(*d, cands[0]);
    if (ws_bytes < extra + conv2d_workspace_bytes(cands[0]))   // workspace sizes are multiples of 256
        return fail(SAMD_ENOSPC, "workspace %zu bytes < %zu needed for the model's plan", ws_bytes,
                    extra + conv2d_workspace_bytes(cands[0]));
    // candidates' workspaces below, the second output and its counter above a 256-byte
    // aligned boundary (the caller's size need not be a multiple of anything)
    const size_t room = (ws_bytes - extra) / 256 * 256;
    std::vector<Conv2dGeom> fit;
    for (const Conv2dGeom &c : cands)
        if (conv2d_workspace_bytes(c) <= room) fit.push_back(c);
    int32_t *y_alt = (int32_t *)((char *)ws + room);
    int32_t *mismatches = (int32_t *)((char *)ws + room + extra - 256);
    const int64_t ny = (int64_t)d->N * d->M * cands[0].Ho * cands[0].Wo;

    hipEvent_t e0 = nullptr, e1 = nullptr;
    auto cleanup = [&](int status) {
        if (e0) (void)hipEventDestroy(e0);
        if (e1) (void)hipEventDestroy(e1);
        return status;
    };
    auto hip_fail = [&](hipError_t e, const char *what) {
        return fail(SAMD_EHIP, "%s: %s", what, hipGetErrorString(e));
    };
    hipError_t he = hipEventCreate(&e0);
    if (he == hipSuccess) he = hipEventCreate(&e1);
    if (he != hipSuccess) return cleanup(hip_fail(he, "hipEventCreate"));

    // The first pass prepares each candidate, checks its result and times it; the second
    // times every candidate again (each keeps its faster time), so that clock ramps and
    // other transients do not decide.  Before the first pass the model's plan runs untimed
    // for a while to bring the clocks up.
    auto run = [&](const Conv2dGeom &c, int32_t *out, int n) {
        int rs = SAMD_OK;
        for (int r = 0; r < n && !rs; ++r)
            if (spaced || !(rs = launch_conv2d_spread(x, c, ws, stream))) rs = launch_conv2d_multiply(c, out, ws, stream);
        return rs;
    };
    auto timed = [&](const Conv2dGeom &c, int32_t *out, float &ms) {
        hipError_t e = hipEventRecord(e0, stream);
        if (e != hipSuccess) return hip_fail(e, "hipEventRecord");
        int rs = run(c, out, reps);
        if (rs) return rs;
        e = hipEventRecord(e1, stream);
        if (e == hipSuccess) e = hipEventSynchronize(e1);
        if (e == hipSuccess) e = hipEventElapsedTime(&ms, e0, e1);
        return e == hipSuccess ? SAMD_OK : hip_fail(e, "timing");
    };
    std::vector<float> best_of(fit.size(), 0.0f);
    for (int pass = 0; pass < 2; ++pass) {
        for (size_t i = 0; i < fit.size(); ++i) {
            const Conv2dGeom &c = fit[i];
            int32_t *out = i == 0 ? y : y_alt;   // the model's plan writes the reference into y
            if ((st = launch_conv2d_prepare(w, c, ws, stream)) ||
                (spaced && (st = launch_conv2d_spread(x, c, ws, stream))) || (st = run(c, out, 1)))
                return cleanup(st);
            if (pass == 0 && i == 0 && (st = run(c, out, 4 * reps))) return cleanup(st);
            if (pass == 0 && i > 0) {
                // every candidate must reproduce the model plan's result exactly
                if ((st = launch_count_mismatch(y, y_alt, ny, mismatches, stream))) return cleanup(st);
                int32_t host = -1;
                he = hipMemcpyAsync(&host, mismatches, sizeof host, hipMemcpyDeviceToHost, stream);
                if (he == hipSuccess) he = hipStreamSynchronize(stream);
                if (he != hipSuccess) return cleanup(hip_fail(he, "mismatch count"));
                if (host != 0)
                    return cleanup(fail(SAMD_EHIP, "candidate plan %zu (L=%d I=%d rows=%d x %d) differs from the "
                                                   "model's plan in %d outputs", i, c.L, c.I, c.rows_blk, c.mblk,
                                        host));
            }
            float ms = 0.0f;
            if ((st = timed(c, out, ms))) return cleanup(st);
            best_of[i] = pass == 0 ? ms : std::min(best_of[i], ms);
        }
    }
    // a candidate must beat the best so far by 2 %: near-ties keep the higher-ranked plan,
    // so repeated tuning of one shape settles on the same plan
    size_t best = 0;
    for (size_t i = 1; i < fit.size(); ++i)
        if (best_of[i] < best_of[best] * 0.98f) best = i;
    const Conv2dGeom &g = fit[best];
    set_tuned_conv2d(*d, xf, wf, g);
    // leave the workspace prepared for the chosen plan (and y holding its result)
    if ((st = launch_conv2d_prepare(w, g, ws, stream)) || (st = launch_conv2d_spread(x, g, ws, stream)) ||
        (st = launch_conv2d_multiply(g, y, ws, stream)))
        return cleanup(st);
    if (chosen) fill_plan(g, chosen);
    return cleanup(SAMD_OK);
}

}  // namespace

extern "C" {

int samd_conv2d_tune(const uint32_t *x, samd_fmt xf, const uint32_t *w, samd_fmt wf, const samd_conv2d_desc *d,
                     int32_t *y, void *ws, size_t ws_bytes, int32_t candidates, int32_t reps,
                     samd_conv2d_plan *chosen, hipStream_t stream) {
    return tune_impl(x, xf, w, wf, d, y, ws, ws_bytes, candidates, reps, chosen, stream, 0);
}

int samd_conv2d_spaced_tune(const uint32_t *x, samd_fmt xf, const uint32_t *w, samd_fmt wf,
                            const samd_conv2d_desc *d, int32_t *y, void *ws, size_t ws_bytes, int32_t candidates,
                            int32_t reps, samd_conv2d_plan *chosen, hipStream_t stream) {
    return tune_impl(x, xf, w, wf, d, y, ws, ws_bytes, candidates, reps, chosen, stream, 1);
}

int samd_conv2d_use_plan(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf, const samd_conv2d_plan *plan) {
    set_error("");
    int st = check_tune_args(d, xf, wf, 1);
    if (st) return st;
    if (!plan) return fail(SAMD_EINVAL, "plan must not be NULL");
    const samd_conv2d_plan want = *plan;
    Conv2dGeom g;
    std::string err;
    st = find_conv2d_candidate(
        *d, xf, wf,
        [&](const Conv2dGeom &c) {
            return c.L == want.lane_bits && c.I == want.lanes && c.xoff == want.x_offset &&
                   c.rows_path == want.shared_rows && c.rh == want.rows_per_thread &&
                   c.rows_blk == want.rows_per_block && c.mblk == want.mblock && c.ks == want.split_waves &&
                   c.spacer == want.spacer_msb;
        },
        g, err, want.layout_spaced ? 1 : 0);
    if (st) return fail(st, "%s", err.c_str());
    set_tuned_conv2d(*d, xf, wf, g);
    return SAMD_OK;
}

int samd_conv2d_untune(const samd_conv2d_desc *d, samd_fmt xf, samd_fmt wf) {
    set_error("");
    if (d) {
        int st = check_fmt(xf, "xf");
        if (!st) st = check_fmt(wf, "wf");
        if (!st) st = check_conv2d_desc(d);
        if (st) return st;
    }
    clear_tuned_conv2d(d, xf, wf);
    return SAMD_OK;
}

}  // extern "C"

// ---- group-scaled rows ----------------------------------------------------------------

namespace {

int64_t type_size(int32_t type) { return type == SAMD_F32 ? 4 : 2; }

int check_type(int32_t type) {
    if (type != SAMD_F32 && type != SAMD_F16 && type != SAMD_BF16)
        return fail(SAMD_EINVAL, "type %d is not SAMD_F32, SAMD_F16 or SAMD_BF16", type);
    return SAMD_OK;
}

int check_group(samd_fmt f, int32_t group, bool weights) {
    int st = check_fmt(f, "fmt");
    if (st) return st;
    if (f.bits != 4 && (weights || f.bits != 8))
        return fail(SAMD_EUNSUPPORTED, "group-scaled %s of %d bits", weights ? "weights" : "rows", f.bits);
    if (group != 32 && group != 64 && group != 128)
        return fail(SAMD_EUNSUPPORTED, "group = %d is not 32, 64 or 128", group);
    return SAMD_OK;
}

int check_size(int64_t n, int64_t least, const char *name) {
    if (n < least || n > INT32_MAX)
        return fail(SAMD_EINVAL, "%s = %lld is outside %lld..2^31 - 1", name, (long long)n, (long long)least);
    return SAMD_OK;
}

// A float matrix: pointer, alignment to its element, row stride.
int check_matrix(const void *p, int32_t type, int64_t rows, int64_t cols, int64_t ld, const char *name) {
    if (!p) return fail(SAMD_EINVAL, "%s must not be NULL", name);
    if ((uintptr_t)p & (type_size(type) - 1)) return fail(SAMD_EALIGN, "%s is not aligned to its elements", name);
    if (ld < cols) return fail(SAMD_EINVAL, "the row stride of %s, %lld, is below its %lld columns", name, (long long)ld,
                               (long long)cols);
    if (rows > 1 && ld > INT64_MAX / 8 / rows)
        return fail(SAMD_EINVAL, "the row stride of %s, %lld, is too large", name, (long long)ld);
    return SAMD_OK;
}

int check_rows(const GroupW &w, samd_fmt f, const char *name) {
    if (!w.q || !w.scale) return fail(SAMD_EINVAL, "the words and scales of %s must not be NULL", name);
    if (f.is_signed ? w.zero != nullptr : w.zero == nullptr)
        return fail(SAMD_EINVAL, f.is_signed ? "%s is signed and takes no zero points" : "%s is unsigned and needs zero points",
                    name);
    if (!aligned4(w.q) || !aligned4(w.scale)) return fail(SAMD_EALIGN, "the words or scales of %s are not aligned", name);
    return SAMD_OK;
}

// Rows of weights: a row's length, where a kernel addresses some tens of rows by 32-bit offsets; and the rows that a
// workgroup of the gradient sums over.
int check_row_length(int64_t K) {
    if (K > kMaxGroupCols)
        return fail(SAMD_EUNSUPPORTED, "K = %lld: rows of more than 2^25 weights are not supported", (long long)K);
    return SAMD_OK;
}

int check_row_count(int64_t M) {
    if (M > kMaxGroupCols)
        return fail(SAMD_EUNSUPPORTED, "M = %lld: gradients over more than 2^25 rows are not supported", (long long)M);
    return SAMD_OK;
}

int check_act(int32_t act) {
    if (act != SAMD_ACT_SILU && act != SAMD_ACT_GELU)
        return fail(SAMD_EINVAL, "act %d is not SAMD_ACT_SILU or SAMD_ACT_GELU", act);
    return SAMD_OK;
}

}  // namespace

extern "C" {

int samd_group_quantize(const void *src, int32_t type, int64_t rows, int64_t cols, int64_t ld, samd_fmt f,
                        int32_t group, uint32_t *q, float *scale, uint8_t *zero, hipStream_t stream) {
    set_error("");
    int st = check_type(type);
    if (!st) st = check_group(f, group, false);
    if (!st) st = check_size(rows, 0, "rows");
    if (!st) st = check_size(cols, 0, "cols");
    if (st) return st;
    if (rows == 0 || cols == 0) return SAMD_OK;
    st = check_matrix(src, type, rows, cols, ld, "src");
    if (!st) st = check_rows({q, scale, zero}, f, "the result");
    if (st) return st;
    return launch_group_quantize(src, type, rows, cols, ld, f, group, q, scale, zero, stream);
}

int samd_group_dequantize(const uint32_t *q, const float *scale, const uint8_t *zero, int64_t rows, int64_t cols,
                          samd_fmt f, int32_t group, void *dst, int32_t type, int64_t ld, hipStream_t stream) {
    set_error("");
    int st = check_type(type);
    if (!st) st = check_group(f, group, false);
    if (!st) st = check_size(rows, 0, "rows");
    if (!st) st = check_size(cols, 0, "cols");
    if (st) return st;
    if (rows == 0 || cols == 0) return SAMD_OK;
    st = check_matrix(dst, type, rows, cols, ld, "dst");
    if (!st) st = check_rows({q, scale, zero}, f, "the rows");
    if (st) return st;
    return launch_group_dequantize({q, scale, zero}, rows, cols, f, group, dst, type, ld, stream);
}

int samd_group_matmul(const void *x, int32_t type, int64_t ldx, const uint32_t *q, const float *scale,
                      const uint8_t *zero, samd_fmt wf, int32_t group, int64_t T, int64_t M, int64_t K, void *y,
                      int64_t ldy, hipStream_t stream) {
    set_error("");
    int st = check_type(type);
    if (!st) st = check_group(wf, group, true);
    if (!st) st = check_size(T, 0, "T");
    if (!st) st = check_size(M, 0, "M");
    if (!st) st = check_size(K, 1, "K");
    if (!st) st = check_row_length(K);
    if (st) return st;
    if (T == 0 || M == 0) return SAMD_OK;
    st = check_matrix(x, type, T, K, ldx, "x");
    if (!st) st = check_matrix(y, type, T, M, ldy, "y");
    if (!st) st = check_rows({q, scale, zero}, wf, "the weights");
    if (st) return st;
    GroupProduct p{};
    p.x = x, p.type = type, p.ldx = ldx, p.w[0] = {q, scale, zero}, p.group = group, p.act = -1;
    p.T = (int32_t)T, p.M = (int32_t)M, p.K = (int32_t)K, p.y = y, p.ldy = ldy;
    return launch_group_product(p, stream);
}

int samd_group_matmul_grad(const void *dy, int32_t type, int64_t lddy, const uint32_t *q, const float *scale,
                           const uint8_t *zero, const void *dy2, const uint32_t *q2, const float *scale2,
                           const uint8_t *zero2, samd_fmt wf, int32_t group, int64_t T, int64_t M, int64_t K,
                           void *dx, int64_t lddx, hipStream_t stream) {
    set_error("");
    int st = check_type(type);
    if (!st) st = check_group(wf, group, true);
    if (!st) st = check_size(T, 0, "T");
    if (!st) st = check_size(M, 1, "M");
    if (!st) st = check_size(K, 0, "K");
    if (!st) st = check_row_length(K);
    if (!st) st = check_row_count(M);
    if (st) return st;
    if (T == 0 || K == 0) return SAMD_OK;
    const bool two = dy2 || q2 || scale2 || zero2;
    st = check_matrix(dy, type, T, M, lddy, "dy");
    if (!st) st = check_matrix(dx, type, T, K, lddx, "dx");
    if (!st) st = check_rows({q, scale, zero}, wf, "the weights");
    if (!st && two) st = check_matrix(dy2, type, T, M, lddy, "dy2");
    if (!st && two) st = check_rows({q2, scale2, zero2}, wf, "the second weights");
    if (st) return st;
    return launch_group_matmul_grad({{dy, dy2}, type, lddy, {{q, scale, zero}, {q2, scale2, zero2}}, group, (int32_t)T,
                                     (int32_t)M, (int32_t)K, dx, lddx}, stream);
}

int samd_group_gated(const void *x, int32_t type, int64_t ldx, const uint32_t *qg, const float *scaleg,
                     const uint8_t *zerog, const uint32_t *qu, const float *scaleu, const uint8_t *zerou, samd_fmt wf,
                     int32_t group, int32_t act, int64_t T, int64_t M, int64_t K, void *h, int64_t ldh, uint32_t *g8,
                     float *gscale, uint32_t *u8, float *uscale, hipStream_t stream) {
    set_error("");
    int st = check_type(type);
    if (!st) st = check_group(wf, group, true);
    if (!st) st = check_act(act);
    if (!st) st = check_size(T, 0, "T");
    if (!st) st = check_size(M, 0, "M");
    if (!st) st = check_size(K, 1, "K");
    if (!st) st = check_row_length(K);
    if (st) return st;
    if (T == 0 || M == 0) return SAMD_OK;
    const bool save = g8 || gscale || u8 || uscale;
    st = check_matrix(x, type, T, K, ldx, "x");
    if (!st) st = check_matrix(h, type, T, M, ldh, "h");
    if (!st) st = check_rows({qg, scaleg, zerog}, wf, "the gate's weights");
    if (!st) st = check_rows({qu, scaleu, zerou}, wf, "the other weights");
    if (!st && save) st = check_rows({g8, gscale, nullptr}, {8, 1}, "the stored gate");
    if (!st && save) st = check_rows({u8, uscale, nullptr}, {8, 1}, "the other stored projection");
    if (st) return st;
    return launch_group_product({x, type, ldx, {{qg, scaleg, zerog}, {qu, scaleu, zerou}}, group, act, (int32_t)T,
                                 (int32_t)M, (int32_t)K, h, ldh, g8, u8, gscale, uscale}, stream);
}

int samd_group_gated_grad(const void *dh, int32_t type, int64_t lddh, const uint32_t *g8, const float *gscale,
                          const uint32_t *u8, const float *uscale, int32_t group, int32_t act, int64_t T, int64_t M,
                          void *dg, void *du, int64_t ldd, hipStream_t stream) {
    set_error("");
    int st = check_type(type);
    if (!st) st = check_group({8, 1}, group, false);
    if (!st) st = check_act(act);
    if (!st) st = check_size(T, 0, "T");
    if (!st) st = check_size(M, 0, "M");
    if (st) return st;
    if (T == 0 || M == 0) return SAMD_OK;
    st = check_matrix(dh, type, T, M, lddh, "dh");
    if (!st) st = check_matrix(dg, type, T, M, ldd, "dg");
    if (!st) st = check_matrix(du, type, T, M, ldd, "du");
    if (!st) st = check_rows({g8, gscale, nullptr}, {8, 1}, "the stored gate");
    if (!st) st = check_rows({u8, uscale, nullptr}, {8, 1}, "the other stored projection");
    if (st) return st;
    return launch_group_gated_grad(dh, type, lddh, {g8, gscale, nullptr}, {u8, uscale, nullptr}, group, act, T, M, dg,
                                   du, ldd, stream);
}

}  // extern "C"
