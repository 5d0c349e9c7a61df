// C entry points of the layers around the step: argument checks, workspace
// layout and the launches. Everything is checked before the first launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <initializer_list>

#include "dion2.h"
#include "dion2_host.h"
#include "layers.h"

using namespace dion2;

static_assert(ACT_NONE == DION2_ACT_NONE && ACT_RELU == DION2_ACT_RELU && ACT_GELU == DION2_ACT_GELU &&
              ACT_GELU_TANH == DION2_ACT_GELU_TANH && ACT_SILU == DION2_ACT_SILU, "one numbering of activations");

namespace {

// C++ exceptions (memory for an error message or a workspace entry) end at
// the C boundary.
template <typename F>
int guarded(F&& f) noexcept {
    try {
        return f();
    } catch (const std::exception&) {
        return DION2_ERR_WORKSPACE;
    } catch (...) {
        return DION2_ERR_HIP;
    }
}

size_t item(int dtype) { return dtype == DION2_DTYPE_BF16 ? 2 : 4; }

dion2_layer_options options_of(const dion2_layer_options* opt) {
    dion2_layer_options o;
    if (opt) o = *opt;
    else dion2_layer_options_init(&o);
    return o;
}

// One argument: a matrix of `rows` rows of `width` entries, `ld` apart.
struct Mat {
    const char* name;
    const void* p;
    int64_t rows, width, ld;
    size_t e;       // bytes an entry
    bool needed;
    size_t align;   // of the pointer
};

int64_t pitch(int64_t ld, int64_t width) { return ld ? ld : width; }
// of a product's operand: a single row's does not matter
int64_t row_pitch(int64_t rows, int64_t ld, int64_t width) { return rows > 1 ? ld : width; }

int check_mat(const Mat& m) {
    if (!m.p) {
        if (m.needed && m.rows > 0) return fail(DION2_ERR_INVALID_ARG, "%s must not be NULL", m.name);
        return DION2_OK;
    }
    if (reinterpret_cast<uintptr_t>(m.p) % m.align)
        return fail(DION2_ERR_INVALID_ARG, "%s must be %zu-byte aligned", m.name, m.align);
    if (m.ld < m.width || m.ld >= (m.rows > 1 ? int64_t(1) << 28 : int64_t(1) << 31))
        return fail(DION2_ERR_INVALID_ARG, "the pitch of %s, %lld, must be at least its width %lld and below 2^28",
                    m.name, (long long)m.ld, (long long)m.width);
    return DION2_OK;
}

bool overlap(const Mat& a, const Mat& b) {
    if (!a.p || !b.p || !a.rows || !b.rows || !a.width || !b.width) return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const uintptr_t ea = pa + ((a.rows - 1) * a.ld + a.width) * a.e, eb = pb + ((b.rows - 1) * b.ld + b.width) * b.e;
    if (ea <= pb || eb <= pa) return false;
    // slices of one buffer: with equal row distances, rows that fall into
    // disjoint columns of it
    const uintptr_t row = (uintptr_t)a.ld * a.e;
    if (row == (uintptr_t)b.ld * b.e) {
        const uintptr_t d = pa <= pb ? (pb - pa) % row : (row - (pa - pb) % row) % row;   // b's columns behind a's
        if (d >= a.width * a.e && d + b.width * b.e <= row) return false;
    }
    return true;
}

bool same(const Mat& a, const Mat& b) { return a.p == b.p && a.ld == b.ld && a.width == b.width && a.e == b.e; }

// Every argument by itself, then every output against every input (which it
// may be exactly where `in_place`) and against the other outputs.
int check_mats(std::initializer_list<Mat> outs, std::initializer_list<Mat> ins, std::initializer_list<const char*> in_place = {}) {
    for (auto* list : {&outs, &ins})
        for (const Mat& m : *list) {
            int st = check_mat(m);
            if (st != DION2_OK) return st;
        }
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        for (const Mat& i : ins) {
            if (!overlap(*o, i)) continue;
            bool allowed = false;
            if (o == outs.begin() && same(*o, i))
                for (const char* n : in_place) allowed = allowed || std::strcmp(n, i.name) == 0;
            if (!allowed) return fail(DION2_ERR_INVALID_ARG, "%s overlaps %s", o->name, i.name);
        }
        for (auto q = o + 1; q != outs.end(); ++q)
            if (overlap(*o, *q)) return fail(DION2_ERR_INVALID_ARG, "%s overlaps %s", o->name, q->name);
    }
    return DION2_OK;
}

int check_options(const dion2_layer_options& o) {
    for (int d : {o.dtype, o.p_dtype, o.g_dtype})
        if (d != DION2_DTYPE_F32 && d != DION2_DTYPE_BF16) return fail(DION2_ERR_INVALID_ARG, "unknown dtype %d", d);
    if (o.act < DION2_ACT_NONE || o.act > DION2_ACT_SILU) return fail(DION2_ERR_INVALID_ARG, "unknown activation %d", o.act);
    if (!(o.eps >= 0.0f) || !std::isfinite(o.eps)) return fail(DION2_ERR_INVALID_ARG, "eps must be finite and >= 0");
    return DION2_OK;
}

int check_sizes(int64_t tokens, int64_t rows, int64_t cols) {
    if (tokens < 0) return fail(DION2_ERR_INVALID_ARG, "tokens must be >= 0, got %lld", (long long)tokens);
    if (rows < 1 || cols < 1)
        return fail(DION2_ERR_INVALID_ARG, "rows, cols must be >= 1, got %lld x %lld", (long long)rows, (long long)cols);
    if (tokens >= (int64_t(1) << 31))
        return fail(DION2_ERR_UNSUPPORTED, "tokens of %lld: below 2^31 are supported", (long long)tokens);
    if (rows > kMaxDim || cols > kMaxDim || rows * cols >= (int64_t(1) << 31))
        return fail(DION2_ERR_UNSUPPORTED, "%lld x %lld: sides up to 2^20 and below 2^31 entries are supported",
                    (long long)rows, (long long)cols);
    // a launch's threads are counted in 32 bits: 256 for a tile of 64 x 64
    const int64_t width = std::max(rows, cols);
    if (((tokens + 63) / 64) * ((width + 63) / 64) >= (int64_t(1) << 24))
        return fail(DION2_ERR_UNSUPPORTED, "%lld tokens of %lld entries are more than one launch takes", (long long)tokens,
                    (long long)width);
    return DION2_OK;
}

// The workspace of a call: the caller's, or the library's unless the stream
// is being captured.
struct Scratch {
    WorkspaceLease lease;
    char* p = nullptr;
};
int take_scratch(const dion2_layer_options& o, size_t bytes, hipStream_t s, Scratch* out) {
    if (o.workspace) {
        if (reinterpret_cast<uintptr_t>(o.workspace) & 255u)
            return fail(DION2_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
        if (o.workspace_bytes < bytes)
            return fail(DION2_ERR_WORKSPACE, "workspace of %zu bytes is below the %zu needed", o.workspace_bytes, bytes);
        out->p = static_cast<char*>(o.workspace);
        return DION2_OK;
    }
    if (!bytes) return DION2_OK;
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    hipError_t e = hipStreamIsCapturing(s, &cap);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if (cap != hipStreamCaptureStatusNone)
        return fail(DION2_ERR_WORKSPACE, "a captured call needs the caller's workspace (%zu bytes)", bytes);
    int st = lease_layer_workspace(s, bytes, &out->lease);
    out->p = out->lease.dev;
    return st;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

int run_product(Product kind, ProductArgs& a, const dion2_layer_options& o, hipStream_t s) {
    a.bf16 = o.dtype == DION2_DTYPE_BF16;
    Scratch ws;
    int st = take_scratch(o, product_workspace(kind, a), s, &ws);
    if (st != DION2_OK) return st;
    a.part = reinterpret_cast<float*>(ws.p);
    hipError_t e = launch_product(kind, a, s);
    return e == hipSuccess ? DION2_OK : hip_fail(e, "launch of a linear layer's product");
}

int linear_forward(void* Y, const void* X, const void* W, const void* bias, const void* R, void* Z, int64_t tokens,
                   int64_t rows, int64_t cols, const dion2_layer_options& o, hipStream_t s) {
    int st = check_options(o);
    if (st == DION2_OK) st = check_sizes(tokens, rows, cols);
    if (st != DION2_OK) return st;
    const size_t e = item(o.dtype), pe = item(o.p_dtype);
    const int64_t ldx = pitch(o.ld_x, cols), ldy = pitch(o.ld_y, rows), ldz = pitch(o.ld_z, rows), ldr = pitch(o.ld_r, rows);
    st = check_mats({{"Y", Y, tokens, rows, ldy, e, true, e}, {"Z", Z, tokens, rows, ldz, e, false, e}},
                    {{"X", X, tokens, cols, ldx, e, true, e},
                     {"W", W, rows, cols, cols, e, true, 16},
                     {"bias", bias, 1, rows, rows, pe, false, pe},
                     {"R", R, tokens, rows, ldr, e, false, e}},
                    {"R"});
    if (st != DION2_OK || tokens == 0) return st;
    ProductArgs a{};
    a.A = X; a.lda = row_pitch(tokens, ldx, cols);
    a.B = W; a.ldb = cols;
    a.M = tokens; a.N = rows; a.K = cols;
    a.out = Y; a.ldo = ldy;
    a.bias = bias; a.bias_bf16 = o.p_dtype == DION2_DTYPE_BF16;
    a.R = R; a.ldr = ldr;
    a.Z = Z; a.ldz = ldz;
    a.act = o.act;
    return run_product(PROD_FORWARD, a, o, s);
}

int linear_backward_input(void* dX, const void* dY, const void* W, const void* Z, int64_t tokens, int64_t rows,
                          int64_t cols, const dion2_layer_options& o, hipStream_t s) {
    int st = check_options(o);
    if (st == DION2_OK) st = check_sizes(tokens, rows, cols);
    if (st != DION2_OK) return st;
    const size_t e = item(o.dtype);
    const bool act = o.act != DION2_ACT_NONE;
    const int64_t lddx = pitch(o.ld_dx, cols), lddy = pitch(o.ld_dy, rows), ldz = pitch(o.ld_z, cols);
    if (!act && Z) return fail(DION2_ERR_INVALID_ARG, "Z is given without an activation");
    st = check_mats({{"dX", dX, tokens, cols, lddx, e, true, e}},
                    {{"dY", dY, tokens, rows, lddy, e, true, e},
                     {"W", W, rows, cols, cols, e, true, 16},
                     {"Z", Z, tokens, cols, ldz, e, act, e}},
                    {"Z"});
    if (st != DION2_OK || tokens == 0) return st;
    ProductArgs a{};
    a.A = dY; a.lda = row_pitch(tokens, lddy, rows);
    a.B = W; a.ldb = cols;
    a.M = tokens; a.N = cols; a.K = rows;
    a.out = dX; a.ldo = lddx;
    a.Z = const_cast<void*>(Z); a.ldz = ldz;
    a.act = o.act;
    return run_product(PROD_INPUT, a, o, s);
}

int linear_backward_weight(void* G, void* dbias, const void* dY, const void* X, int64_t tokens, int64_t rows,
                           int64_t cols, const dion2_layer_options& o, hipStream_t s) {
    int st = check_options(o);
    if (st == DION2_OK) st = check_sizes(tokens, rows, cols);
    if (st != DION2_OK) return st;
    const size_t e = item(o.dtype), ge = item(o.g_dtype);
    if (!G && !dbias) return fail(DION2_ERR_INVALID_ARG, "G and dbias must not both be NULL");
    const int64_t lddy = pitch(o.ld_dy, rows), ldx = pitch(o.ld_x, cols);
    st = check_mats({{"G", G, rows, cols, cols, ge, false, 16}, {"dbias", dbias, 1, rows, rows, ge, false, ge}},
                    {{"dY", dY, tokens, rows, lddy, e, true, e}, {"X", X, tokens, cols, ldx, e, G != nullptr, e}});
    if (st != DION2_OK) return st;
    ColSumArgs c{};
    c.X = dY; c.ldx = lddy; c.tokens = tokens; c.width = rows;
    c.bf16 = o.dtype == DION2_DTYPE_BF16;
    c.out = dbias; c.out_bf16 = o.g_dtype == DION2_DTYPE_BF16; c.accumulate = o.accumulate != 0;
    ProductArgs a{};
    a.A = dY; a.lda = row_pitch(tokens, lddy, rows);
    a.B = X; a.ldb = row_pitch(tokens, ldx, cols);
    a.M = rows; a.N = cols; a.K = tokens;
    a.out = G; a.ldo = cols; a.out_bf16 = c.out_bf16;
    a.accumulate = c.accumulate;
    a.bf16 = c.bf16;
    // the bias gradient's partial sums come out of the product where its form
    // gives them, else out of a pass of their own
    const int64_t beside = G && dbias ? product_row_sums(a) : 0;
    c.blocks = beside ? beside : col_sum_blocks(tokens, rows);
    const size_t part = G ? align256(product_workspace(PROD_WEIGHT, a)) : 0;
    Scratch ws;
    st = take_scratch(o, part + (dbias ? align256((size_t)c.blocks * rows * 4) : 0), s, &ws);
    if (st != DION2_OK) return st;
    c.part = reinterpret_cast<float*>(ws.p + part);
    hipError_t err = hipSuccess;
    if (G) {
        a.part = reinterpret_cast<float*>(ws.p);
        a.row_sums = beside ? c.part : nullptr;
        err = launch_product(PROD_WEIGHT, a, s);
        if (err != hipSuccess) return hip_fail(err, "launch of a linear layer's product");
    }
    if (dbias) err = beside ? launch_col_join(c, s) : launch_col_sum(c, s);
    return err == hipSuccess ? DION2_OK : hip_fail(err, "launch of the bias gradient");
}

int activation_backward(void* dZ, const void* dY, const void* Z, int64_t tokens, int64_t width,
                        const dion2_layer_options& o, hipStream_t s) {
    int st = check_options(o);
    if (st == DION2_OK) st = check_sizes(tokens, 1, width);
    if (st != DION2_OK) return st;
    const size_t e = item(o.dtype);
    ActGradArgs a{};
    a.ldo = pitch(o.ld_dz, width); a.ldy = pitch(o.ld_dy, width); a.ldz = pitch(o.ld_z, width);
    st = check_mats({{"dZ", dZ, tokens, width, a.ldo, e, true, e}},
                    {{"dY", dY, tokens, width, a.ldy, e, true, e}, {"Z", Z, tokens, width, a.ldz, e, true, e}}, {"dY", "Z"});
    if (st != DION2_OK || tokens == 0) return st;
    a.dY = dY; a.Z = Z; a.dZ = dZ;
    a.tokens = tokens; a.width = width;
    a.act = o.act; a.bf16 = o.dtype == DION2_DTYPE_BF16;
    hipError_t err = launch_act_grad(a, s);
    return err == hipSuccess ? DION2_OK : hip_fail(err, "launch of an activation's gradient");
}

int layernorm_forward(void* Y, float* mean, float* rstd, const void* X, const void* gamma, const void* beta,
                      int64_t tokens, int64_t cols, const dion2_layer_options& o, hipStream_t s) {
    int st = check_options(o);
    if (st == DION2_OK) st = check_sizes(tokens, 1, cols);
    if (st != DION2_OK) return st;
    const size_t e = item(o.dtype), pe = item(o.p_dtype);
    NormArgs a{};
    a.ldx = pitch(o.ld_x, cols); a.ldy = pitch(o.ld_y, cols);
    st = check_mats({{"Y", Y, tokens, cols, a.ldy, e, true, e},
                     {"mean", mean, 1, tokens, tokens, 4, false, 4},
                     {"rstd", rstd, 1, tokens, tokens, 4, false, 4}},
                    {{"X", X, tokens, cols, a.ldx, e, true, e},
                     {"gamma", gamma, 1, cols, cols, pe, false, pe},
                     {"beta", beta, 1, cols, cols, pe, false, pe}},
                    {"X"});
    if (st != DION2_OK || tokens == 0) return st;
    a.X = X; a.gamma = gamma; a.beta = beta; a.Y = Y; a.mean = mean; a.rstd = rstd;
    a.tokens = tokens; a.cols = cols; a.eps = o.eps;
    a.bf16 = o.dtype == DION2_DTYPE_BF16; a.p_bf16 = o.p_dtype == DION2_DTYPE_BF16;
    hipError_t err = launch_norm(a, s);
    return err == hipSuccess ? DION2_OK : hip_fail(err, "launch of layer norm");
}

int layernorm_backward(void* dX, void* dgamma, void* dbeta, const void* dY, const void* X, const float* mean,
                       const float* rstd, const void* gamma, const void* dR, int64_t tokens, int64_t cols,
                       const dion2_layer_options& o, hipStream_t s) {
    int st = check_options(o);
    if (st == DION2_OK) st = check_sizes(tokens, 1, cols);
    if (st != DION2_OK) return st;
    if (!dX && !dgamma && !dbeta) return fail(DION2_ERR_INVALID_ARG, "dX, dgamma and dbeta must not all be NULL");
    if (!dX && dR) return fail(DION2_ERR_INVALID_ARG, "dR is given without dX");
    const size_t e = item(o.dtype), pe = item(o.p_dtype), ge = item(o.g_dtype);
    NormGradArgs a{};
    a.lddx = pitch(o.ld_dx, cols); a.lddy = pitch(o.ld_dy, cols); a.ldx = pitch(o.ld_x, cols); a.lddr = pitch(o.ld_dr, cols);
    st = check_mats({{"dX", dX, tokens, cols, a.lddx, e, false, e},
                     {"dgamma", dgamma, 1, cols, cols, ge, false, ge},
                     {"dbeta", dbeta, 1, cols, cols, ge, false, ge}},
                    {{"dY", dY, tokens, cols, a.lddy, e, true, e},
                     {"X", X, tokens, cols, a.ldx, e, true, e},
                     {"mean", mean, tokens ? 1 : 0, tokens, tokens, 4, true, 4},
                     {"rstd", rstd, tokens ? 1 : 0, tokens, tokens, 4, true, 4},
                     {"gamma", gamma, 1, cols, cols, pe, false, pe},
                     {"dR", dR, tokens, cols, a.lddr, e, false, e}},
                    {"dY", "X", "dR"});
    if (st != DION2_OK) return st;
    a.dY = dY; a.X = X; a.mean = mean; a.rstd = rstd; a.gamma = gamma; a.dR = dR;
    a.dX = dX; a.dgamma = dgamma; a.dbeta = dbeta;
    a.tokens = tokens; a.cols = cols;
    a.bf16 = o.dtype == DION2_DTYPE_BF16; a.p_bf16 = o.p_dtype == DION2_DTYPE_BF16;
    a.g_bf16 = o.g_dtype == DION2_DTYPE_BF16; a.accumulate = o.accumulate != 0;
    a.blocks = norm_grad_blocks(tokens, cols, a.bf16);
    Scratch ws;
    st = take_scratch(o, dgamma || dbeta ? align256((size_t)a.blocks * 2 * cols * 4) : 0, s, &ws);
    if (st != DION2_OK) return st;
    a.part = reinterpret_cast<float*>(ws.p);
    hipError_t err = launch_norm_grad(a, s);
    return err == hipSuccess ? DION2_OK : hip_fail(err, "launch of layer norm's gradient");
}

}  // namespace

extern "C" {

void dion2_layer_options_init(dion2_layer_options* opt) {
    if (!opt) return;
    std::memset(opt, 0, sizeof *opt);
    opt->dtype = opt->p_dtype = opt->g_dtype = DION2_DTYPE_BF16;
    opt->act = DION2_ACT_NONE;
    opt->eps = 1e-5f;
}

int dion2_linear_forward(void* Y, const void* X, const void* W, const void* bias, const void* R, void* Z, int64_t tokens,
                         int64_t rows, int64_t cols, const dion2_layer_options* opt, void* stream) {
    return guarded([&] {
        return linear_forward(Y, X, W, bias, R, Z, tokens, rows, cols, options_of(opt), static_cast<hipStream_t>(stream));
    });
}

int dion2_linear_backward_input(void* dX, const void* dY, const void* W, const void* Z, int64_t tokens, int64_t rows,
                                int64_t cols, const dion2_layer_options* opt, void* stream) {
    return guarded([&] {
        return linear_backward_input(dX, dY, W, Z, tokens, rows, cols, options_of(opt), static_cast<hipStream_t>(stream));
    });
}

int dion2_linear_backward_weight(void* G, void* dbias, const void* dY, const void* X, int64_t tokens, int64_t rows,
                                 int64_t cols, const dion2_layer_options* opt, void* stream) {
    return guarded([&] {
        return linear_backward_weight(G, dbias, dY, X, tokens, rows, cols, options_of(opt), static_cast<hipStream_t>(stream));
    });
}

int dion2_activation_backward(void* dZ, const void* dY, const void* Z, int64_t tokens, int64_t width,
                              const dion2_layer_options* opt, void* stream) {
    return guarded([&] { return activation_backward(dZ, dY, Z, tokens, width, options_of(opt), static_cast<hipStream_t>(stream)); });
}

int dion2_layernorm_forward(void* Y, float* mean, float* rstd, const void* X, const void* gamma, const void* beta,
                            int64_t tokens, int64_t cols, const dion2_layer_options* opt, void* stream) {
    return guarded([&] {
        return layernorm_forward(Y, mean, rstd, X, gamma, beta, tokens, cols, options_of(opt), static_cast<hipStream_t>(stream));
    });
}

int dion2_layernorm_backward(void* dX, void* dgamma, void* dbeta, const void* dY, const void* X, const float* mean,
                             const float* rstd, const void* gamma, const void* dR, int64_t tokens, int64_t cols,
                             const dion2_layer_options* opt, void* stream) {
    return guarded([&] {
        return layernorm_backward(dX, dgamma, dbeta, dY, X, mean, rstd, gamma, dR, tokens, cols, options_of(opt),
                                  static_cast<hipStream_t>(stream));
    });
}

size_t dion2_linear_workspace_size(int64_t tokens, int64_t rows, int64_t cols, const dion2_layer_options* opt) try {
    const dion2_layer_options o = options_of(opt);
    if (check_options(o) != DION2_OK || check_sizes(tokens, rows, cols) != DION2_OK) return 0;
    ProductArgs f{}, i{}, w{};
    f.bf16 = i.bf16 = w.bf16 = o.dtype == DION2_DTYPE_BF16;
    f.lda = w.ldb = row_pitch(tokens, pitch(o.ld_x, cols), cols);
    i.lda = w.lda = row_pitch(tokens, pitch(o.ld_dy, rows), rows);
    f.ldb = i.ldb = cols;
    f.M = tokens; f.N = rows; f.K = cols;
    i.M = tokens; i.N = cols; i.K = rows;
    w.M = rows; w.N = cols; w.K = tokens;
    return std::max({align256(product_workspace_most(PROD_FORWARD, f)), align256(product_workspace_most(PROD_INPUT, i)),
                     align256(product_workspace_most(PROD_WEIGHT, w)) + align256((size_t)col_sum_blocks(tokens, rows) * rows * 4)});
} catch (const std::exception&) {
    return 0;
}

size_t dion2_layernorm_workspace_size(int64_t tokens, int64_t cols, const dion2_layer_options* opt) try {
    const dion2_layer_options o = options_of(opt);
    if (check_options(o) != DION2_OK || check_sizes(tokens, 1, cols) != DION2_OK) return 0;
    return align256((size_t)norm_grad_blocks(tokens, cols, o.dtype == DION2_DTYPE_BF16) * 2 * cols * 4);
} catch (const std::exception&) {
    return 0;
}

}  // extern "C"
