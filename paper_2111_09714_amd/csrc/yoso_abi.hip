// C ABI of libyoso: argument validation, workspace sizing and dispatch.
// Every check runs on the host before the first HIP call.
#include <float.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <mutex>

#include "../../include/yoso.h"
#include "launch.h"

// Workspace of yoso_backward_noalloc: one copy of this array per GPU the library
// runs on, held until the process ends.  Host code never uses the name itself
// (on the host it is only a stand-in for the device symbol): it asks
// hipGetSymbolAddress for each device's address once and passes that pointer.
constexpr size_t kNoAllocScratchBytes = size_t{64} << 20;
__device__ __align__(256) unsigned char scratch[kNoAllocScratchBytes];

namespace {

thread_local char g_last_error[512] = "";

yoso_status fail(yoso_status s, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof g_last_error, fmt, ap);
    va_end(ap);
    return s;
}

yoso_status device_status(hipError_t e, const char *what) {
    if (e == hipSuccess) return YOSO_OK;
    return fail(YOSO_ERR_DEVICE, "%s: %s (%s)", what, hipGetErrorName(e), hipGetErrorString(e));
}

#define YOSO_TRY(expr)                         \
    do {                                       \
        const yoso_status _s = (expr);         \
        if (_s != YOSO_OK) return _s;          \
    } while (0)

constexpr int64_t kMaxN = 65536;
constexpr int64_t kMaxGrid = 0x7fffffff;

yoso_status check_dtype(yoso_dtype dt) {
    if (dt != YOSO_F32 && dt != YOSO_BF16) return fail(YOSO_ERR_DTYPE, "unknown dtype %d", (int)dt);
    return YOSO_OK;
}

yoso_status check_shape(int64_t bh, int64_t n_q, int64_t n_k, int32_t d, int32_t m) {
    if (d != 64) return fail(YOSO_ERR_SHAPE, "d = %d; only d = 64 is supported", d);
    if (bh < 0) return fail(YOSO_ERR_SHAPE, "bh = %lld < 0", (long long)bh);
    if (n_q < 0 || n_q > kMaxN) return fail(YOSO_ERR_SHAPE, "n_q = %lld outside [0, 65536]", (long long)n_q);
    if (n_k < 0 || n_k > kMaxN) return fail(YOSO_ERR_SHAPE, "n_k = %lld outside [0, 65536]", (long long)n_k);
    // grid limits: 2*bh*m sort and pair blocks, bh*32 table blocks, bh*n/16 reduce blocks
    if (m > 0 && bh > kMaxGrid / (2 * (int64_t)m))
        return fail(YOSO_ERR_SHAPE, "bh = %lld too large for m = %d", (long long)bh, m);
    if (bh > kMaxGrid / 64) return fail(YOSO_ERR_SHAPE, "bh = %lld too large", (long long)bh);
    const int64_t nmax = n_q > n_k ? n_q : n_k;
    if (nmax > 0 && bh > kMaxGrid * 16 / nmax)
        return fail(YOSO_ERR_SHAPE, "bh*n = %lld*%lld too large", (long long)bh, (long long)nmax);
    return YOSO_OK;
}

// row operations: any number of 64-value rows (grid-stride kernels)
yoso_status check_rows(int64_t rows, int32_t d) {
    if (d != 64) return fail(YOSO_ERR_SHAPE, "d = %d; only d = 64 is supported", d);
    if (rows < 0) return fail(YOSO_ERR_SHAPE, "rows = %lld < 0", (long long)rows);
    if (rows > (int64_t{1} << 40)) return fail(YOSO_ERR_SHAPE, "rows = %lld too large", (long long)rows);
    return YOSO_OK;
}

yoso_status check_hash(int32_t m, int32_t tau) {
    if (tau < 1 || tau > 12) return fail(YOSO_ERR_TAU, "tau = %d outside [1, 12]", tau);
    if (m < 1 || m > 64) return fail(YOSO_ERR_TAU, "m = %d outside [1, 64]", m);
    if (m * tau > 512) return fail(YOSO_ERR_TAU, "m*tau = %d > 512", m * tau);
    return YOSO_OK;
}

yoso_status check_ptr(const void *p, int64_t elems, const char *name) {
    if (elems == 0) return YOSO_OK;
    if (p == nullptr) return fail(YOSO_ERR_NULL, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & 15u) return fail(YOSO_ERR_ALIGN, "%s is not 16-byte aligned", name);
    return YOSO_OK;
}

// row operations on rows of any width up to kMaxWidth
constexpr int32_t kMaxWidth = 8192;

yoso_status check_width(int32_t d) {
    if (d < 1 || d > kMaxWidth) return fail(YOSO_ERR_SHAPE, "d = %d outside [1, %d]", d, kMaxWidth);
    return YOSO_OK;
}

yoso_status check_layer_norm(int64_t rows, int32_t d) {
    YOSO_TRY(check_width(d));
    if (rows < 0) return fail(YOSO_ERR_SHAPE, "rows = %lld < 0", (long long)rows);
    if (rows > (int64_t{1} << 40)) return fail(YOSO_ERR_SHAPE, "rows = %lld too large", (long long)rows);
    return YOSO_OK;
}

yoso_status check_eps(float eps) {
    if (!(eps >= FLT_MIN) || !isfinite(eps))
        return fail(YOSO_ERR_VALUE, "eps = %g is not a positive normal number", (double)eps);
    return YOSO_OK;
}

// (the gradient sorts tokens by the upper bits of their ids into at most 2048 buckets of at most 512 ids)
constexpr int64_t kMaxTokens = int64_t{1} << 27, kMaxVocab = int64_t{1} << 20;

yoso_status check_embedding(int64_t tokens, int64_t n_pos, int64_t vocab, int32_t d) {
    YOSO_TRY(check_width(d));
    if (tokens < 0 || tokens > kMaxTokens)
        return fail(YOSO_ERR_SHAPE, "tokens = %lld outside [0, 2^27]", (long long)tokens);
    if (vocab < 1 || vocab > kMaxVocab) return fail(YOSO_ERR_SHAPE, "vocab = %lld outside [1, 2^20]", (long long)vocab);
    if (n_pos < 0 || n_pos > kMaxTokens)
        return fail(YOSO_ERR_SHAPE, "n_pos = %lld outside [0, 2^27]", (long long)n_pos);
    if (n_pos > 0 && tokens % n_pos != 0)
        return fail(YOSO_ERR_SHAPE, "n_pos = %lld does not divide tokens = %lld", (long long)n_pos, (long long)tokens);
    return YOSO_OK;
}

yoso_status check_index(yoso_index type) {
    if (type != YOSO_I32 && type != YOSO_I64) return fail(YOSO_ERR_DTYPE, "unknown index type %d", (int)type);
    return YOSO_OK;
}

// token ids are read one by one: any whole element (a serving loop passes single tokens of a longer tensor)
yoso_status check_ids(const void *ids, int64_t tokens, yoso_index type) {
    if (tokens == 0) return YOSO_OK;
    if (ids == nullptr) return fail(YOSO_ERR_NULL, "ids is NULL");
    if (reinterpret_cast<uintptr_t>(ids) & (type == YOSO_I64 ? 7u : 3u))
        return fail(YOSO_ERR_ALIGN, "ids is not aligned to its elements");
    return YOSO_OK;
}

// Rows of d values: 16-byte aligned where they are whole 16-byte vectors; others start at any element
// (so that rows can be cut out of a tensor).  NULL where there are none, or where optional.
yoso_status check_row_ptr(const void *p, int64_t rows, int32_t d, yoso_dtype dtype, const char *name, bool optional = false) {
    if (rows == 0 || (optional && p == nullptr)) return YOSO_OK;
    if (p == nullptr) return fail(YOSO_ERR_NULL, "%s is NULL", name);
    const unsigned size = dtype == YOSO_BF16 ? 2 : 4, align = d * size % 16 == 0 ? 16 : size;
    if (reinterpret_cast<uintptr_t>(p) & (align - 1)) return fail(YOSO_ERR_ALIGN, "%s is not %u-byte aligned", name, align);
    return YOSO_OK;
}

// an optional fp32 parameter vector
yoso_status check_param(const float *p, const char *name) {
    if (reinterpret_cast<uintptr_t>(p) & 3u) return fail(YOSO_ERR_ALIGN, "%s is not 4-byte aligned", name);
    return YOSO_OK;
}

size_t required_workspace(yoso_op op, bool bf16, int64_t bh, int64_t n_q, int64_t n_k, int32_t m, int32_t tau) {
    switch (op) {
        case YOSO_OP_HASH: return 0;
        case YOSO_OP_FORWARD:
            return yoso::dense_forward_applies(bh, n_q, n_k, m, tau) ? 0 : yoso::table_workspace_bytes(bf16, bh, n_q, m, tau);
        case YOSO_OP_BACKWARD: return yoso::backward_layout(bf16, bh, n_q, n_k, m, tau).total;
        case YOSO_OP_BACKWARD_STAR: return yoso::backward_star_layout(bf16, bh, n_q, n_k, m, tau).total;
    }
    return 0;
}

yoso_status check_workspace(const void *ws, size_t have, size_t need) {
    if (need == 0) return YOSO_OK;
    if (ws == nullptr) return fail(YOSO_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", need);
    if (have < need) return fail(YOSO_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
    if (reinterpret_cast<uintptr_t>(ws) & 15u) return fail(YOSO_ERR_ALIGN, "workspace is not 16-byte aligned");
    return YOSO_OK;
}

// The scratch array's address on the device of `stream` (which must be the
// current device), looked up on the first call on that device.
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void *g_scratch_ptr[kMaxDevices] = {};

yoso_status scratch_for(hipStream_t stream, void **ptr) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return device_status(e, "hipGetDevice");
    if (stream != nullptr) {
        int sdev = 0;
        if ((e = hipStreamGetDevice(stream, &sdev)) != hipSuccess) return device_status(e, "hipStreamGetDevice");
        if (sdev != dev)
            return fail(YOSO_ERR_DEVICE, "the stream belongs to device %d but device %d is current", sdev, dev);
    }
    if (dev < 0 || dev >= kMaxDevices) return fail(YOSO_ERR_DEVICE, "device %d beyond the %d supported", dev, kMaxDevices);
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (g_scratch_ptr[dev] == nullptr) {
        void *p = nullptr;
        if ((e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch))) != hipSuccess)
            return device_status(e, "hipGetSymbolAddress(scratch)");
        g_scratch_ptr[dev] = p;
    }
    *ptr = g_scratch_ptr[dev];
    return YOSO_OK;
}

}  // namespace

extern "C" {

const char *yoso_status_str(yoso_status status) {
    switch (status) {
        case YOSO_OK: return "ok";
        case YOSO_ERR_NULL: return "null pointer";
        case YOSO_ERR_SHAPE: return "unsupported shape";
        case YOSO_ERR_TAU: return "tau or m out of range";
        case YOSO_ERR_DTYPE: return "unknown dtype";
        case YOSO_ERR_ALIGN: return "misaligned pointer";
        case YOSO_ERR_WORKSPACE: return "workspace missing or too small";
        case YOSO_ERR_DEVICE: return "HIP error";
        case YOSO_ERR_OP: return "unknown op";
        case YOSO_ERR_VALUE: return "argument value not accepted";
    }
    return "unknown status";
}

const char *yoso_last_error(void) { return g_last_error; }

size_t yoso_workspace_bytes(int op, int64_t bh, int64_t n_q, int64_t n_k, int32_t d, int32_t m, int32_t tau,
                            yoso_dtype dtype) {
    g_last_error[0] = '\0';
    const size_t bad = static_cast<size_t>(-1);
    if (op != YOSO_OP_HASH && op != YOSO_OP_FORWARD && op != YOSO_OP_BACKWARD && op != YOSO_OP_BACKWARD_STAR) {
        fail(YOSO_ERR_OP, "unknown op %d", op);
        return bad;
    }
    if (check_dtype(dtype) != YOSO_OK || check_shape(bh, n_q, n_k, d, m) != YOSO_OK || check_hash(m, tau) != YOSO_OK)
        return bad;
    return required_workspace(static_cast<yoso_op>(op), dtype == YOSO_BF16, bh, n_q, n_k, m, tau);
}

yoso_status yoso_hash(const void *x, yoso_dtype dtype, int64_t bh, int64_t n, int32_t d, const float *R,
                      int32_t m, int32_t tau, uint16_t *codes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n, 0, d, m));
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(x, bh * n * d, "x"));
    YOSO_TRY(check_ptr(R, (int64_t)d * m * tau, "R"));
    YOSO_TRY(check_ptr(codes, bh * n * m, "codes"));
    return device_status(yoso::launch_hash(x, dtype == YOSO_BF16, bh, n, R, m, tau, codes,
                                           static_cast<hipStream_t>(stream)),
                         "yoso_hash");
}

yoso_status yoso_fast_hyperplanes(const uint64_t *signs, int32_t d, int32_t m, int32_t tau, float *R,
                                  void *stream) {
    g_last_error[0] = '\0';
    if (d != 64) return fail(YOSO_ERR_SHAPE, "d = %d; only d = 64 is supported", d);
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(signs, 3 * (((int64_t)m * tau + 63) / 64), "signs"));
    YOSO_TRY(check_ptr(R, (int64_t)d * m * tau, "R"));
    return device_status(yoso::launch_fast_hyperplanes(signs, m, tau, R, static_cast<hipStream_t>(stream)),
                         "yoso_fast_hyperplanes");
}

yoso_status yoso_fast_hash(const void *x, yoso_dtype dtype, int64_t bh, int64_t n, int32_t d,
                           const uint64_t *signs, int32_t m, int32_t tau, uint16_t *codes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n, 0, d, m));
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(x, bh * n * d, "x"));
    YOSO_TRY(check_ptr(signs, 3 * (((int64_t)m * tau + 63) / 64), "signs"));
    YOSO_TRY(check_ptr(codes, bh * n * m, "codes"));
    return device_status(yoso::launch_fast_hash(x, dtype == YOSO_BF16, bh, n, signs, m, tau, codes,
                                                static_cast<hipStream_t>(stream)),
                         "yoso_fast_hash");
}

yoso_status yoso_forward(const uint16_t *qcodes, const uint16_t *kcodes, const void *v, yoso_dtype dtype,
                         int64_t bh, int64_t n_q, int64_t n_k, int32_t d, int32_t m, int32_t tau, void *y,
                         void *workspace, size_t workspace_bytes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n_q, n_k, d, m));
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(qcodes, bh * m * n_q, "qcodes"));
    YOSO_TRY(check_ptr(kcodes, bh * m * n_k, "kcodes"));
    YOSO_TRY(check_ptr(v, bh * n_k * d, "v"));
    YOSO_TRY(check_ptr(y, bh * n_q * d, "y"));
    const bool bf16 = dtype == YOSO_BF16;
    YOSO_TRY(check_workspace(workspace, workspace_bytes, required_workspace(YOSO_OP_FORWARD, bf16, bh, n_q, n_k, m, tau)));
    if (yoso::tile_forward_applies(bf16, bh, n_q, n_k, m, tau) && yoso::tile_forward_codes(qcodes, kcodes, m, tau))
        return device_status(yoso::launch_tile_forward(qcodes, kcodes, v, y, bf16, bh, n_q, n_k, m, tau,
                                                       static_cast<hipStream_t>(stream)),
                             "yoso_forward");
    if (yoso::dense_forward_applies(bh, n_q, n_k, m, tau))
        return device_status(yoso::launch_dense_forward(qcodes, kcodes, v, y, bf16, bh, n_q, n_k, m, tau,
                                                        static_cast<hipStream_t>(stream)),
                             "yoso_forward");
    return device_status(yoso::launch_table(kcodes, v, qcodes, y, bf16, bh, n_k, n_q, m, tau, workspace,
                                            static_cast<hipStream_t>(stream)),
                         "yoso_forward");
}

yoso_status yoso_backward(const uint16_t *qcodes, const uint16_t *kcodes, const void *q, const void *k,
                          const void *v, const void *dy, yoso_dtype dtype, int64_t bh, int64_t n_q, int64_t n_k,
                          int32_t d, int32_t m, int32_t tau, void *dq, void *dk, void *dv, void *workspace,
                          size_t workspace_bytes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n_q, n_k, d, m));
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(qcodes, bh * m * n_q, "qcodes"));
    YOSO_TRY(check_ptr(kcodes, bh * m * n_k, "kcodes"));
    YOSO_TRY(check_ptr(q, bh * n_q * d, "q"));
    YOSO_TRY(check_ptr(k, bh * n_k * d, "k"));
    YOSO_TRY(check_ptr(v, bh * n_k * d, "v"));
    YOSO_TRY(check_ptr(dy, bh * n_q * d, "dy"));
    YOSO_TRY(check_ptr(dq, bh * n_q * d, "dq"));
    YOSO_TRY(check_ptr(dk, bh * n_k * d, "dk"));
    YOSO_TRY(check_ptr(dv, bh * n_k * d, "dv"));
    const bool bf16 = dtype == YOSO_BF16;
    YOSO_TRY(check_workspace(workspace, workspace_bytes, required_workspace(YOSO_OP_BACKWARD, bf16, bh, n_q, n_k, m, tau)));
    return device_status(yoso::launch_backward(qcodes, kcodes, q, k, v, dy, bf16, bh, n_q, n_k, m, tau, dq, dk, dv,
                                               workspace, static_cast<hipStream_t>(stream)),
                         "yoso_backward");
}

yoso_status yoso_backward_star(const uint16_t *qcodes, const uint16_t *kcodes, const void *q, const void *k,
                               const void *v, const void *dy, yoso_dtype dtype, int64_t bh, int64_t n_q, int64_t n_k,
                               int32_t d, int32_t m, int32_t tau, void *dq, void *dk, void *dv, void *workspace,
                               size_t workspace_bytes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n_q, n_k, d, m * tau));
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(qcodes, bh * m * n_q, "qcodes"));
    YOSO_TRY(check_ptr(kcodes, bh * m * n_k, "kcodes"));
    YOSO_TRY(check_ptr(q, bh * n_q * d, "q"));
    YOSO_TRY(check_ptr(k, bh * n_k * d, "k"));
    YOSO_TRY(check_ptr(v, bh * n_k * d, "v"));
    YOSO_TRY(check_ptr(dy, bh * n_q * d, "dy"));
    YOSO_TRY(check_ptr(dq, bh * n_q * d, "dq"));
    YOSO_TRY(check_ptr(dk, bh * n_k * d, "dk"));
    YOSO_TRY(check_ptr(dv, bh * n_k * d, "dv"));
    const bool bf16 = dtype == YOSO_BF16;
    YOSO_TRY(check_workspace(workspace, workspace_bytes,
                             required_workspace(YOSO_OP_BACKWARD_STAR, bf16, bh, n_q, n_k, m, tau)));
    return device_status(yoso::launch_backward_star(qcodes, kcodes, q, k, v, dy, bf16, bh, n_q, n_k, m, tau, dq, dk,
                                                    dv, workspace, static_cast<hipStream_t>(stream)),
                         "yoso_backward_star");
}

yoso_status yoso_backward_noalloc(const uint16_t *qcodes, const uint16_t *kcodes, const void *q, const void *k,
                                  const void *v, const void *dy, yoso_dtype dtype, int64_t bh, int64_t n_q,
                                  int64_t n_k, int32_t d, int32_t m, int32_t tau, void *dq, void *dk, void *dv,
                                  void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n_q, n_k, d, m));
    YOSO_TRY(check_hash(m, tau));
    YOSO_TRY(check_ptr(qcodes, bh * m * n_q, "qcodes"));
    YOSO_TRY(check_ptr(kcodes, bh * m * n_k, "kcodes"));
    YOSO_TRY(check_ptr(q, bh * n_q * d, "q"));
    YOSO_TRY(check_ptr(k, bh * n_k * d, "k"));
    YOSO_TRY(check_ptr(v, bh * n_k * d, "v"));
    YOSO_TRY(check_ptr(dy, bh * n_q * d, "dy"));
    YOSO_TRY(check_ptr(dq, bh * n_q * d, "dq"));
    YOSO_TRY(check_ptr(dk, bh * n_k * d, "dk"));
    YOSO_TRY(check_ptr(dv, bh * n_k * d, "dv"));
    const bool bf16 = dtype == YOSO_BF16;
    const size_t need = required_workspace(YOSO_OP_BACKWARD, bf16, bh, n_q, n_k, m, tau);
    if (need > kNoAllocScratchBytes)
        return fail(YOSO_ERR_WORKSPACE,
                    "these shapes need %zu bytes of scratch; yoso_backward_noalloc has %zu (use yoso_backward with a "
                    "workspace)",
                    need, kNoAllocScratchBytes);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    void *ws = nullptr;
    if (need > 0) YOSO_TRY(scratch_for(s, &ws));
    return device_status(yoso::launch_backward(qcodes, kcodes, q, k, v, dy, bf16, bh, n_q, n_k, m, tau, dq, dk, dv,
                                               ws, s),
                         "yoso_backward_noalloc");
}

size_t yoso_backward_noalloc_limit(void) { return kNoAllocScratchBytes; }

int32_t yoso_backward_table_threshold(void) { return yoso::backward_table_threshold(); }

yoso_status yoso_l2_normalize(const void *x, yoso_dtype dtype, int64_t rows, int32_t d, void *y, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_rows(rows, d));
    YOSO_TRY(check_ptr(x, rows * d, "x"));
    YOSO_TRY(check_ptr(y, rows * d, "y"));
    return device_status(yoso::launch_l2norm(x, y, dtype == YOSO_BF16, rows, static_cast<hipStream_t>(stream)),
                         "yoso_l2_normalize");
}

yoso_status yoso_l2_normalize_backward(const void *x, const void *dy, yoso_dtype dtype, int64_t rows, int32_t d,
                                       void *dx, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_rows(rows, d));
    YOSO_TRY(check_ptr(x, rows * d, "x"));
    YOSO_TRY(check_ptr(dy, rows * d, "dy"));
    YOSO_TRY(check_ptr(dx, rows * d, "dx"));
    return device_status(
        yoso::launch_l2norm_backward(x, dy, dx, dtype == YOSO_BF16, rows, static_cast<hipStream_t>(stream)),
        "yoso_l2_normalize_backward");
}

size_t yoso_layer_norm_backward_workspace_bytes(int64_t rows, int32_t d, yoso_dtype dtype) {
    g_last_error[0] = '\0';
    if (check_dtype(dtype) != YOSO_OK || check_layer_norm(rows, d) != YOSO_OK) return static_cast<size_t>(-1);
    return yoso::layer_norm_backward_workspace(dtype == YOSO_BF16, rows, d);
}

yoso_status yoso_layer_norm(const void *x, const void *residual, const float *weight, const float *bias,
                            yoso_dtype dtype, int64_t rows, int32_t d, float eps, void *sum, void *y, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_layer_norm(rows, d));
    YOSO_TRY(check_eps(eps));
    YOSO_TRY(check_row_ptr(x, rows, d, dtype, "x"));
    YOSO_TRY(check_row_ptr(residual, rows, d, dtype, "residual", true));
    YOSO_TRY(check_param(weight, "weight"));
    YOSO_TRY(check_param(bias, "bias"));
    YOSO_TRY(check_row_ptr(sum, rows, d, dtype, "sum", true));
    YOSO_TRY(check_row_ptr(y, rows, d, dtype, "y"));
    if (sum != nullptr && sum == y) return fail(YOSO_ERR_VALUE, "sum and y are one buffer");
    const yoso::LayerNorm a{x, residual, weight, bias, rows, d, eps, sum, y};
    return device_status(yoso::launch_layer_norm(a, dtype == YOSO_BF16, static_cast<hipStream_t>(stream)),
                         "yoso_layer_norm");
}

yoso_status yoso_layer_norm_backward(const void *z, const float *weight, const void *dy, const void *dsum,
                                     yoso_dtype dtype, int64_t rows, int32_t d, float eps, void *dx, float *dweight,
                                     float *dbias, void *workspace, size_t workspace_bytes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_layer_norm(rows, d));
    YOSO_TRY(check_eps(eps));
    YOSO_TRY(check_row_ptr(z, rows, d, dtype, "z"));
    YOSO_TRY(check_param(weight, "weight"));
    YOSO_TRY(check_row_ptr(dy, rows, d, dtype, "dy"));
    YOSO_TRY(check_row_ptr(dsum, rows, d, dtype, "dsum", true));
    YOSO_TRY(check_row_ptr(dx, rows, d, dtype, "dx"));
    if ((dweight == nullptr) != (dbias == nullptr))
        return fail(YOSO_ERR_NULL, "%s is NULL: dweight and dbias are given together", dweight ? "dbias" : "dweight");
    YOSO_TRY(check_param(dweight, "dweight"));
    YOSO_TRY(check_param(dbias, "dbias"));
    if (dweight != nullptr && dweight == dbias) return fail(YOSO_ERR_VALUE, "dweight and dbias are one buffer");
    const bool bf16 = dtype == YOSO_BF16;
    if (dweight)
        YOSO_TRY(check_workspace(workspace, workspace_bytes, yoso::layer_norm_backward_workspace(bf16, rows, d)));
    const yoso::LayerNormBackward a{z, weight, dy, dsum, rows, d, eps, dx, dweight, dbias, workspace};
    return device_status(yoso::launch_layer_norm_backward(a, bf16, static_cast<hipStream_t>(stream)),
                         "yoso_layer_norm_backward");
}

size_t yoso_embedding_backward_workspace_bytes(int64_t tokens, int64_t n_pos, int64_t vocab, int32_t d,
                                               yoso_dtype dtype) {
    g_last_error[0] = '\0';
    if (check_dtype(dtype) != YOSO_OK || check_embedding(tokens, n_pos, vocab, d) != YOSO_OK)
        return static_cast<size_t>(-1);
    return yoso::embedding_backward_workspace(dtype == YOSO_BF16, tokens, n_pos, vocab, d);
}

yoso_status yoso_embedding(const void *ids, yoso_index index, const void *table, const void *pos, yoso_dtype dtype,
                           int64_t tokens, int64_t n_pos, int64_t vocab, int32_t d, float scale, void *y,
                           void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_index(index));
    YOSO_TRY(check_embedding(tokens, n_pos, vocab, d));
    if (!isfinite(scale)) return fail(YOSO_ERR_VALUE, "scale = %g is not finite", (double)scale);
    YOSO_TRY(check_ids(ids, tokens, index));
    YOSO_TRY(check_row_ptr(table, tokens, d, dtype, "table"));
    if (pos != nullptr && n_pos == 0) return fail(YOSO_ERR_SHAPE, "pos is given but n_pos = 0");
    YOSO_TRY(check_row_ptr(pos, n_pos, d, dtype, "pos"));
    YOSO_TRY(check_row_ptr(y, tokens, d, dtype, "y"));
    const yoso::Embedding a{ids, table, pos, tokens, n_pos, vocab, d, scale, y};
    return device_status(
        yoso::launch_embedding(a, dtype == YOSO_BF16, index == YOSO_I64, static_cast<hipStream_t>(stream)),
        "yoso_embedding");
}

yoso_status yoso_embedding_backward(const void *ids, yoso_index index, const void *dy, yoso_dtype dtype,
                                    int64_t tokens, int64_t n_pos, int64_t vocab, int32_t d, float scale,
                                    void *dtable, void *dpos, void *workspace, size_t workspace_bytes, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_index(index));
    YOSO_TRY(check_embedding(tokens, n_pos, vocab, d));
    if (!isfinite(scale)) return fail(YOSO_ERR_VALUE, "scale = %g is not finite", (double)scale);
    YOSO_TRY(check_ids(ids, tokens, index));
    YOSO_TRY(check_row_ptr(dy, tokens, d, dtype, "dy"));
    YOSO_TRY(check_row_ptr(dtable, vocab, d, dtype, "dtable"));
    if (dpos != nullptr && n_pos == 0) return fail(YOSO_ERR_SHAPE, "dpos is given but n_pos = 0");
    YOSO_TRY(check_row_ptr(dpos, n_pos, d, dtype, "dpos"));
    const bool bf16 = dtype == YOSO_BF16;
    YOSO_TRY(check_workspace(workspace, workspace_bytes,
                             yoso::embedding_backward_workspace(bf16, tokens, n_pos, vocab, d)));
    const yoso::EmbeddingBackward a{ids, dy, tokens, n_pos, vocab, d, scale, dtable, dpos, workspace};
    return device_status(
        yoso::launch_embedding_backward(a, bf16, index == YOSO_I64, static_cast<hipStream_t>(stream)),
        "yoso_embedding_backward");
}

yoso_status yoso_expectation_forward(const void *q, const void *k, const void *v, yoso_dtype dtype, int64_t bh,
                                     int64_t n_q, int64_t n_k, int32_t d, int32_t tau, void *y, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n_q, n_k, d, 1));
    YOSO_TRY(check_hash(1, tau));
    YOSO_TRY(check_ptr(q, bh * n_q * d, "q"));
    YOSO_TRY(check_ptr(k, bh * n_k * d, "k"));
    YOSO_TRY(check_ptr(v, bh * n_k * d, "v"));
    YOSO_TRY(check_ptr(y, bh * n_q * d, "y"));
    return device_status(yoso::launch_expect_forward(q, k, v, y, dtype == YOSO_BF16, bh, n_q, n_k, tau,
                                                     static_cast<hipStream_t>(stream)),
                         "yoso_expectation_forward");
}

yoso_status yoso_expectation_backward(const void *q, const void *k, const void *v, const void *dy, yoso_dtype dtype,
                                      int64_t bh, int64_t n_q, int64_t n_k, int32_t d, int32_t tau, void *dq,
                                      void *dk, void *dv, void *stream) {
    g_last_error[0] = '\0';
    YOSO_TRY(check_dtype(dtype));
    YOSO_TRY(check_shape(bh, n_q, n_k, d, 1));
    YOSO_TRY(check_hash(1, tau));
    YOSO_TRY(check_ptr(q, bh * n_q * d, "q"));
    YOSO_TRY(check_ptr(k, bh * n_k * d, "k"));
    YOSO_TRY(check_ptr(v, bh * n_k * d, "v"));
    YOSO_TRY(check_ptr(dy, bh * n_q * d, "dy"));
    YOSO_TRY(check_ptr(dq, bh * n_q * d, "dq"));
    YOSO_TRY(check_ptr(dk, bh * n_k * d, "dk"));
    YOSO_TRY(check_ptr(dv, bh * n_k * d, "dv"));
    return device_status(yoso::launch_expect_backward(q, k, v, dy, dq, dk, dv, dtype == YOSO_BF16, bh, n_q, n_k, tau,
                                                      static_cast<hipStream_t>(stream)),
                         "yoso_expectation_backward");
}

}  // extern "C"
