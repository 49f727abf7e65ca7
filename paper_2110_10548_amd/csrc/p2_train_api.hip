// C entry points of include/p2_train.h: checks of arguments, workspaces, launches.  Nothing here waits or allocates.
#include <algorithm>
#include <cmath>
#include <exception>
#include <limits>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 40;
constexpr int64_t kMostSide = (int64_t)1 << 17;
constexpr int64_t kMostMatrices = 65535;
constexpr int32_t kMostSteps = 64;

int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

bool known_type(int32_t t) { return t == P2_F32 || t == P2_BF16 || t == P2_F16; }

// Whether `p` may hold elements of `bytes` each.
bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// A matrix argument with rows: nullptr where it is fine, else what is wrong with it.
const char* bad_rows(const void* p, int32_t type, int64_t stride, int64_t rows, int64_t cols) {
    if (rows > 0 && !p) return "null argument";
    if (!aligned_to(p, type_bytes(type))) return "pointer not aligned to its elements";
    if (stride < cols) return "rows overlap: stride smaller than the row";
    if (rows > 1 && stride > std::numeric_limits<int64_t>::max() / 8 / rows) return "matrix larger than the address space";
    return nullptr;
}

// Runs an entry point's body; what the host throws comes back as an error.
template <typename F> int32_t guarded(F&& body) {
    try {
        return body();
    } catch (const std::exception& e) {
        return api_fail(P2_EDEVICE, std::string("host failure: ") + e.what());
    } catch (...) {
        return api_fail(P2_EDEVICE, "host failure");
    }
}

int32_t launched(hipError_t e, const char* what) { return e == hipSuccess ? P2_OK : api_hip_fail(e, what); }

int32_t check_norm(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return api_fail(P2_EINVAL, "rows < 0 or cols < 1");
    if (rows > kMostRows || cols > ((int64_t)1 << 31) - 1) return api_fail(P2_EUNSUPPORTED, "more than 2^40 rows or 2^31 - 1 columns");
    return P2_OK;
}

int32_t check_balance(int64_t tokens, int32_t experts, int32_t k) {
    if (tokens < 0 || experts < 1 || k < 1) return api_fail(P2_EINVAL, "tokens < 0, experts < 1 or k < 1");
    if (k > experts) return api_fail(P2_EINVAL, "k larger than the number of experts");
    if (experts > P2_MAX_EXPERTS || k > P2_MAX_CHOSEN) return api_fail(P2_EUNSUPPORTED, "more than 1024 experts, or 64 of them a token");
    if (tokens > ((int64_t)1 << 34)) return api_fail(P2_EUNSUPPORTED, "more than 2^34 tokens");
    return P2_OK;
}

int32_t check_matrices(int64_t count, int64_t rows, int64_t cols) {
    if (count < 0 || rows < 1 || cols < 1) return api_fail(P2_EINVAL, "count < 0, rows < 1 or cols < 1");
    if (rows > kMostSide || cols > kMostSide || count > kMostMatrices) return api_fail(P2_EUNSUPPORTED, "sides longer than 2^17, or more than 65535 matrices");
    if ((double)orthogonalize_workspace(1, rows, cols) * (double)std::max<int64_t>(count, 1) >= std::ldexp(1.0, 40))
        return api_fail(P2_EUNSUPPORTED, "a workspace of 2^40 bytes or more");
    return P2_OK;
}

struct BalanceRoom { int64_t prob, count, ticket, bytes; };
BalanceRoom balance_room(int64_t tokens, int32_t experts) {
    const int64_t lines = balance_forward_partials(tokens, experts);
    BalanceRoom r = {};
    if (lines == 1) return r;                  // one block keeps its sums to itself
    r.prob = 0;
    r.count = round256(lines * experts * 4);
    r.ticket = r.count + round256(lines * (experts + 1) * 4);
    r.bytes = r.ticket + 256;
    return r;
}

}  // namespace

}  // namespace p2

using namespace p2;

extern "C" {

int32_t p2_layer_norm_forward(const void* x, int32_t type, int64_t x_stride, const void* weight, const void* bias, int32_t weight_type,
                              int64_t rows, int64_t cols, double eps, void* y, int64_t y_stride, float* mean, float* rstd, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type) || !known_type(weight_type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_norm(rows, cols);
        if (rc != P2_OK) return rc;
        if (!(eps >= 0.0) || std::isinf(eps)) return api_fail(P2_EINVAL, "eps must be >= 0");
        for (const char* bad : {bad_rows(x, type, x_stride, rows, cols), bad_rows(y, type, y_stride, rows, cols)})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (y == x && rows > 1 && y_stride != x_stride) return api_fail(P2_EINVAL, "y is x with another stride");
        if (!aligned_to(weight, type_bytes(weight_type)) || !aligned_to(bias, type_bytes(weight_type)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
            return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        if (rows == 0) return P2_OK;
        NormForward a = {};
        a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd;
        a.x_stride = x_stride; a.y_stride = y_stride; a.rows = rows; a.cols = cols;
        a.eps = (float)eps; a.type = type; a.weight_type = weight_type;
        return launched(launch_norm_forward(a, (hipStream_t)stream), "layer norm");
    });
}

int32_t p2_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_norm(rows, cols);
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = round256(norm_backward_partials(rows, cols) * 4);
        return P2_OK;
    });
}

int32_t p2_layer_norm_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int32_t type, const void* weight,
                               int32_t weight_type, const float* mean, const float* rstd, int64_t rows, int64_t cols, void* dx, int64_t dx_stride,
                               void* dweight, void* dbias, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type) || !known_type(weight_type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_norm(rows, cols);
        if (rc != P2_OK) return rc;
        for (const char* bad : {bad_rows(dy, type, dy_stride, rows, cols), bad_rows(x, type, x_stride, rows, cols),
                                dx ? bad_rows(dx, type, dx_stride, rows, cols) : nullptr})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (rows > 0 && (!mean || !rstd)) return api_fail(P2_EINVAL, "null argument");
        if (dx && dx == dy && rows > 1 && dx_stride != dy_stride) return api_fail(P2_EINVAL, "dx is dy with another stride");
        for (const void* p : {weight, (const void*)dweight, (const void*)dbias})
            if (!aligned_to(p, type_bytes(weight_type))) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        const bool sums = dweight || dbias;
        if (sums) {
            if (!workspace || !aligned_to(workspace, 256)) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
            if (workspace_bytes < round256(norm_backward_partials(rows, cols) * 4)) return api_fail(P2_ENOSPC, "workspace too small");
        }
        if (!dx && !sums) return P2_OK;
        if (rows == 0 && !sums) return P2_OK;
        NormBackward a = {};
        a.dy = dy; a.x = x; a.weight = weight; a.mean = mean; a.rstd = rstd; a.dx = dx; a.dweight = dweight; a.dbias = dbias;
        a.partial = sums ? static_cast<float*>(workspace) : nullptr;
        a.dy_stride = dy_stride; a.x_stride = x_stride; a.dx_stride = dx_stride; a.rows = rows; a.cols = cols;
        a.type = type; a.weight_type = weight_type;
        return launched(launch_norm_backward(a, (hipStream_t)stream), "layer norm's gradient");
    });
}

int32_t p2_balance_forward_workspace(int64_t tokens, int32_t experts, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_balance(tokens, experts, 1);
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = balance_room(tokens, experts).bytes;
        return P2_OK;
    });
}

int32_t p2_balance_forward(const void* logits, int32_t type, int64_t stride, const uint8_t* keep, int64_t tokens, int32_t experts, int32_t k,
                           int32_t* expert, float* gate, int64_t* counts, float* prob_sum, int64_t* kept, float* loss, void* workspace,
                           int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_balance(tokens, experts, k);
        if (rc != P2_OK) return rc;
        if (const char* bad = bad_rows(logits, type, stride, tokens, experts)) return api_fail(P2_EINVAL, bad);
        if ((tokens > 0 && (!expert || !gate)) || !counts || !prob_sum || !kept || !loss) return api_fail(P2_EINVAL, "null argument");
        if (!aligned_to(expert, 4) || !aligned_to(gate, 4) || !aligned_to(counts, 8) || !aligned_to(prob_sum, 4) || !aligned_to(kept, 8) || !aligned_to(loss, 4))
            return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        const BalanceRoom room = balance_room(tokens, experts);
        if (room.bytes && (!workspace || !aligned_to(workspace, 256))) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < room.bytes) return api_fail(P2_ENOSPC, "workspace too small");
        char* w = static_cast<char*>(workspace);
        BalanceForward a = {};
        a.logits = logits; a.keep = keep; a.expert = expert; a.gate = gate; a.counts = counts; a.prob_sum = prob_sum; a.kept = kept; a.loss = loss;
        a.part_prob = reinterpret_cast<float*>(w + room.prob);
        a.part_count = reinterpret_cast<int32_t*>(w + room.count);
        a.ticket = reinterpret_cast<uint32_t*>(w + room.ticket);
        a.stride = stride; a.tokens = tokens; a.experts = experts; a.k = k; a.type = type;
        return launched(launch_balance_forward(a, (hipStream_t)stream), "balance");
    });
}

int32_t p2_balance_loss(const int64_t* counts, const float* prob_sum, const int64_t* kept, int32_t experts, int32_t k, float* loss, void* stream) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_balance(0, experts, k);
        if (rc != P2_OK) return rc;
        if (!counts || !prob_sum || !kept || !loss) return api_fail(P2_EINVAL, "null argument");
        if (!aligned_to(counts, 8) || !aligned_to(prob_sum, 4) || !aligned_to(kept, 8) || !aligned_to(loss, 4))
            return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        return launched(launch_balance_loss(counts, prob_sum, kept, experts, k, loss, (hipStream_t)stream), "balance loss");
    });
}

int32_t p2_balance_backward(const void* logits, int32_t type, int64_t stride, const uint8_t* keep, int64_t tokens, int32_t experts, int32_t k,
                            const int32_t* expert, const float* dgate, const int64_t* counts, const int64_t* kept, const float* dloss,
                            void* dlogits, int64_t dlogits_stride, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_balance(tokens, experts, k);
        if (rc != P2_OK) return rc;
        for (const char* bad : {bad_rows(logits, type, stride, tokens, experts), bad_rows(dlogits, type, dlogits_stride, tokens, experts)})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (!counts || !kept || (tokens > 0 && dgate && !expert)) return api_fail(P2_EINVAL, "null argument");
        if (dlogits == logits && tokens > 1 && dlogits_stride != stride) return api_fail(P2_EINVAL, "dlogits are the logits with another stride");
        if (!aligned_to(expert, 4) || !aligned_to(dgate, 4) || !aligned_to(counts, 8) || !aligned_to(kept, 8) || !aligned_to(dloss, 4))
            return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        BalanceBackward a = {};
        a.logits = logits; a.keep = keep; a.expert = expert; a.dgate = dgate; a.counts = counts; a.kept = kept; a.dloss = dloss; a.dlogits = dlogits;
        a.stride = stride; a.dlogits_stride = dlogits_stride; a.tokens = tokens; a.experts = experts; a.k = k; a.type = type;
        return launched(launch_balance_backward(a, (hipStream_t)stream), "balance's gradient");
    });
}

int32_t p2_orthogonalize_workspace(int64_t count, int64_t rows, int64_t cols, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_matrices(count, rows, cols);
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = count ? orthogonalize_workspace(count, rows, cols) : 0;
        return P2_OK;
    });
}

int32_t p2_orthogonalize(const void* g, int32_t type, int64_t stride, int64_t matrix_stride, int64_t count, int64_t rows, int64_t cols, int32_t steps,
                         const double* coefficients, double eps, double scale, void* out, int32_t out_type, int64_t out_stride,
                         int64_t out_matrix_stride, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type) || !known_type(out_type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_matrices(count, rows, cols);
        if (rc != P2_OK) return rc;
        if (steps < 1 || steps > kMostSteps) return api_fail(P2_EINVAL, "steps outside 1 to 64");
        if (!coefficients) return api_fail(P2_EINVAL, "null argument");
        for (int i = 0; i < 3; ++i) if (!std::isfinite(coefficients[i])) return api_fail(P2_EINVAL, "coefficients must be finite");
        if (!(eps >= 0.0) || std::isinf(eps) || !std::isfinite(scale)) return api_fail(P2_EINVAL, "eps must be >= 0, scale finite");
        for (const char* bad : {bad_rows(g, type, stride, count * rows, cols), bad_rows(out, out_type, out_stride, count * rows, cols)})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (count > 1 && (matrix_stride < 0 || out_matrix_stride < (rows - 1) * out_stride + cols)) return api_fail(P2_EINVAL, "matrices overlap");
        if (count > 1 && std::max(matrix_stride, out_matrix_stride) > std::numeric_limits<int64_t>::max() / 8 / count)
            return api_fail(P2_EINVAL, "matrix larger than the address space");
        if (count == 0) return P2_OK;
        double bounds[kMostSteps + 1];
        Orthogonalize a = {};
        a.g = g; a.out = out; a.workspace = workspace;
        a.stride = stride; a.matrix_stride = matrix_stride; a.count = count; a.rows = rows; a.cols = cols;
        a.out_stride = out_stride; a.out_matrix_stride = out_matrix_stride;
        a.type = type; a.out_type = out_type; a.steps = steps;
        a.a = coefficients[0]; a.b = coefficients[1]; a.c = coefficients[2]; a.eps = eps; a.scale = scale;
        a.bounds = bounds;
        if (!orthogonalize_bounds(a, bounds)) return api_fail(P2_EUNSUPPORTED, "with these coefficients singular values may pass 2^10");
        const int64_t room = orthogonalize_workspace(count, rows, cols);
        if (room && (!workspace || !aligned_to(workspace, 256))) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < room) return api_fail(P2_ENOSPC, "workspace too small");
        return launched(launch_orthogonalize(a, (hipStream_t)stream), "orthogonalize");
    });
}

}  // extern "C"
