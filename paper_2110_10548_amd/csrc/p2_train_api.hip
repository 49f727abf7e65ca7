// C entry points of include/p2_train.h: checks of arguments, workspaces, launches.  Nothing here waits or allocates.
#include <algorithm>
#include <cmath>
#include <exception>
#include <limits>
#include <utility>
#include <vector>

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

int32_t check_route(int64_t tokens, int32_t experts, int32_t k, int32_t groups) {
    int32_t rc = check_balance(tokens, experts, k);
    if (rc != P2_OK) return rc;
    if (groups < 1 || experts % groups) return api_fail(P2_EINVAL, "experts must be a multiple of groups");
    if (groups > P2_MAX_GROUPS) return api_fail(P2_EUNSUPPORTED, "more than 64 groups");
    return P2_OK;
}
struct RouteRoom { int64_t again, bytes; };
RouteRoom route_room(int64_t tokens, int32_t experts, int32_t k, int32_t groups) {
    const int64_t lines = route_forward_blocks(tokens, experts, k, groups);
    if (lines == 1) return {};
    const int64_t again = round256(lines * (experts + 1) * 4);
    return {again, again + round256(tokens)};
}

// Tensors of a call over many: as many and as long as the kernels count.
constexpr int64_t kMostTensors = (int64_t)1 << 20, kMostValues = (int64_t)1 << 40;
template <typename F> int32_t check_tensors(int64_t n, F&& count) {
    if (n < 0) return api_fail(P2_EINVAL, "n < 0");
    if (n > kMostTensors) return api_fail(P2_EUNSUPPORTED, "more than 2^20 tensors");
    int64_t all = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (count(i) < 0) return api_fail(P2_EINVAL, "a tensor's count < 0");
        if (count(i) > kMostValues || (all += count(i)) > kMostValues) return api_fail(P2_EUNSUPPORTED, "more than 2^40 values");
    }
    return P2_OK;
}

// Whether some of these ranges, all of which are written, overlap.
typedef std::pair<const char*, const char*> Range;
bool overlap(std::vector<Range>& ranges) {
    std::sort(ranges.begin(), ranges.end());
    for (size_t i = 1; i < ranges.size(); ++i)
        if (ranges[i].first < ranges[i - 1].second) return true;
    return false;
}

Range range_of(const void* p, int64_t n, size_t bytes) { return {static_cast<const char*>(p), static_cast<const char*>(p) + (size_t)n * bytes}; }
// Whether one more overlaps these, which are in order and apart.
bool overlap(const std::vector<Range>& ranges, const Range& one) {
    const auto after = std::lower_bound(ranges.begin(), ranges.end(), Range(one.second, nullptr));       // the first that begins at its end or later
    return after != ranges.begin() && std::prev(after)->second > one.first;
}

// A matrix of a product, in bytes.
struct Extent { int64_t at, rows, row, stride; };
Extent extent_of(const void* p, int32_t type, int64_t stride, int64_t rows, int64_t cols) {
    const int64_t size = (int64_t)type_bytes(type);
    return {(int64_t)reinterpret_cast<uintptr_t>(p), p ? rows : 0, cols * size, rows > 1 ? stride * size : 0};
}
// Whether two matrices share bytes.  Of one stride each may have columns of its own in a buffer; of different ones it is by the first and the last byte.
bool overlap(const Extent& a, const Extent& b) {
    if (a.rows <= 0 || b.rows <= 0) return false;
    if (a.at + (a.rows - 1) * a.stride + a.row <= b.at || b.at + (b.rows - 1) * b.stride + b.row <= a.at) return false;
    const int64_t stride = std::max(a.stride, b.stride), off = b.at - a.at;
    if (stride == 0 || (a.stride != b.stride && a.rows > 1 && b.rows > 1)) return true;
    // row i of a and row j of b, i - j = m:  m stride < off + b.row  and  off < m stride + a.row
    const auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
    const int64_t least = std::max(floor_div(off - a.row, stride) + 1, 1 - b.rows), most = std::min(floor_div(off + b.row - 1, stride), a.rows - 1);
    return least <= most;
}

constexpr int64_t kMostLinear = (int64_t)1 << 20;
int32_t check_linear(int32_t type, int64_t rows, int64_t inner, int64_t outer) {
    if (!known_type(type)) return api_fail(P2_EINVAL, "unknown element type");
    if (rows < 0 || inner < 1 || outer < 1) return api_fail(P2_EINVAL, "rows < 0, inner < 1 or outer < 1");
    if (rows > kMostLinear || inner > kMostLinear || outer > kMostLinear) return api_fail(P2_EUNSUPPORTED, "rows, inner or outer more than 2^20");
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

int32_t p2_route_forward_workspace(int64_t tokens, int32_t experts, int32_t k, int32_t groups, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_route(tokens, experts, k, groups);
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = route_room(tokens, experts, k, groups).bytes;
        return P2_OK;
    });
}

int32_t p2_route_forward(const void* logits, int32_t type, int64_t stride, const uint8_t* keep, const float* bias, int64_t tokens, int32_t experts,
                         int32_t k, int32_t score, int32_t groups, int32_t group_limit, int32_t group_best, int32_t renormalise, double scale,
                         int32_t* expert, float* gate, int64_t* counts, int64_t* kept, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_route(tokens, experts, k, groups);
        if (rc != P2_OK) return rc;
        if (score != P2_SOFTMAX && score != P2_SIGMOID) return api_fail(P2_EINVAL, "unknown score");
        if (group_limit < 1 || group_limit > groups) return api_fail(P2_EINVAL, "group_limit outside 1 to groups");
        if (group_best != 1 && group_best != 2) return api_fail(P2_EINVAL, "group_best must be 1 or 2");
        if (!std::isfinite(scale)) return api_fail(P2_EINVAL, "scale must be finite");
        if (const char* bad = bad_rows(logits, type, stride, tokens, experts)) return api_fail(P2_EINVAL, bad);
        if ((tokens > 0 && (!expert || !gate)) || !counts || !kept) return api_fail(P2_EINVAL, "null argument");
        if (!aligned_to(bias, 4) || !aligned_to(expert, 4) || !aligned_to(gate, 4) || !aligned_to(counts, 8) || !aligned_to(kept, 8))
            return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        const RouteRoom room = route_room(tokens, experts, k, groups);
        if (room.bytes && (!workspace || !aligned_to(workspace, 256))) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < room.bytes) return api_fail(P2_ENOSPC, "workspace too small");
        RouteForward a = {};
        a.logits = logits; a.keep = keep; a.bias = bias; a.expert = expert; a.gate = gate; a.counts = counts; a.kept = kept;
        a.part_count = static_cast<int32_t*>(workspace);
        a.again = static_cast<uint8_t*>(workspace) + room.again;
        a.stride = stride; a.tokens = tokens; a.scale = (float)scale; a.experts = experts; a.k = k; a.type = type; a.score = score;
        a.groups = groups; a.group_limit = group_limit; a.group_best = group_best; a.renormalise = renormalise != 0;
        return launched(launch_route_forward(a, (hipStream_t)stream), "route");
    });
}

int32_t p2_route_backward(const void* logits, int32_t type, int64_t stride, int64_t tokens, int32_t experts, int32_t k, int32_t score,
                          int32_t renormalise, double scale, const int32_t* expert, const float* dgate, void* dlogits, int64_t dlogits_stride, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type)) return api_fail(P2_EINVAL, "unknown element type");
        int32_t rc = check_balance(tokens, experts, k);
        if (rc != P2_OK) return rc;
        if (score != P2_SOFTMAX && score != P2_SIGMOID) return api_fail(P2_EINVAL, "unknown score");
        if (!std::isfinite(scale)) return api_fail(P2_EINVAL, "scale must be finite");
        for (const char* bad : {bad_rows(logits, type, stride, tokens, experts), bad_rows(dlogits, type, dlogits_stride, tokens, experts)})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (tokens > 0 && (!expert || !dgate)) return api_fail(P2_EINVAL, "null argument");
        if (dlogits == logits && tokens > 1 && dlogits_stride != stride) return api_fail(P2_EINVAL, "dlogits are the logits with another stride");
        if (!aligned_to(expert, 4) || !aligned_to(dgate, 4)) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        RouteBackward a = {};
        a.logits = logits; a.expert = expert; a.dgate = dgate; a.dlogits = dlogits; a.stride = stride; a.dlogits_stride = dlogits_stride;
        a.tokens = tokens; a.scale = (float)scale; a.experts = experts; a.k = k; a.type = type; a.score = score; a.renormalise = renormalise != 0;
        return launched(launch_route_backward(a, (hipStream_t)stream), "route's gradient");
    });
}

int32_t p2_route_bias(const float* bias, const int64_t* counts, int32_t experts, double rate, float* out, void* stream) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_balance(0, experts, 1);
        if (rc != P2_OK) return rc;
        if (!std::isfinite(rate)) return api_fail(P2_EINVAL, "rate must be finite");
        if (!bias || !counts || !out) return api_fail(P2_EINVAL, "null argument");
        if (!aligned_to(bias, 4) || !aligned_to(counts, 8) || !aligned_to(out, 4)) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        return launched(launch_route_bias(bias, counts, experts, (float)rate, out, (hipStream_t)stream), "route's biases");
    });
}

int32_t p2_square_sum_workspace(int64_t n, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_tensors(n, [](int64_t) { return 0; });
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = round256(square_sum_parts(n) * 8);
        return P2_OK;
    });
}

int32_t p2_square_sum(const void* const* tensors, const int64_t* counts, int64_t n, int32_t type, double* out, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type)) return api_fail(P2_EINVAL, "unknown element type");
        if (n > 0 && (!tensors || !counts)) return api_fail(P2_EINVAL, "null argument");
        int32_t rc = check_tensors(n, [&](int64_t i) { return counts[i]; });
        if (rc != P2_OK) return rc;
        for (int64_t i = 0; i < n; ++i) {
            if (counts[i] > 0 && !tensors[i]) return api_fail(P2_EINVAL, "null argument");
            if (!aligned_to(tensors[i], type_bytes(type))) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        }
        if (!out) return api_fail(P2_EINVAL, "null argument");
        if (!aligned_to(out, 8)) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        if (!workspace || !aligned_to(workspace, 256)) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < round256(square_sum_parts(n) * 8)) return api_fail(P2_ENOSPC, "workspace too small");
        return launched(launch_square_sum(tensors, counts, n, type, out, static_cast<double*>(workspace), (hipStream_t)stream), "sum of squares");
    });
}

int32_t p2_adamw_workspace(int64_t* bytes) {
    return guarded([&]() -> int32_t {
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = 256;
        return P2_OK;
    });
}

int32_t p2_adamw(const p2_adamw_tensor* tensors, int64_t n, int32_t type, int32_t grad_type, int32_t copy_type, int32_t state_bits, int64_t* step,
                 const float* rate, double lr, double beta1, double beta2, double eps, double weight_decay, double grad_factor, const double* square_sum,
                 double max_norm, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        if (!known_type(type) || !known_type(grad_type) || !known_type(copy_type)) return api_fail(P2_EINVAL, "unknown element type");
        if (state_bits != 32 && state_bits != 8) return api_fail(P2_EINVAL, "states have 32 or 8 bits");
        if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return api_fail(P2_EINVAL, "betas must be in [0, 1)");
        if (!std::isfinite(lr) || !std::isfinite(weight_decay)) return api_fail(P2_EINVAL, "lr and weight_decay must be finite");
        if (!(eps >= 0.0) || std::isinf(eps)) return api_fail(P2_EINVAL, "eps must be >= 0");
        if (state_bits == 8 && eps < 1e-12) return api_fail(P2_EUNSUPPORTED, "8-bit states take eps >= 1e-12");
        if (!(grad_factor > 0.0) || std::isinf(grad_factor)) return api_fail(P2_EINVAL, "grad_factor must be > 0");
        if (square_sum && !(max_norm > 0.0)) return api_fail(P2_EINVAL, "max_norm must be > 0");
        if (n > 0 && !tensors) return api_fail(P2_EINVAL, "null argument");
        int32_t rc = check_tensors(n, [&](int64_t i) { return tensors[i].count; });
        if (rc != P2_OK) return rc;
        const size_t size = type_bytes(type), state = state_bits == 8 ? 1 : 4;
        std::vector<Range> written;
        written.reserve((size_t)n * 6);
        for (int64_t i = 0; i < n; ++i) {
            const p2_adamw_tensor& t = tensors[i];
            if (t.count == 0) continue;
            if (!t.param || !t.grad || !t.mean || !t.square) return api_fail(P2_EINVAL, "null argument");
            if (state_bits == 8 && (!t.mean_scale || !t.square_scale)) return api_fail(P2_EINVAL, "8-bit states need their scales");
            if (!aligned_to(t.param, size) || !aligned_to(t.grad, type_bytes(grad_type)) || !aligned_to(t.copy, type_bytes(copy_type)) || !aligned_to(t.mean, state) ||
                !aligned_to(t.square, state) || !aligned_to(t.mean_scale, 4) || !aligned_to(t.square_scale, 4))
                return api_fail(P2_EINVAL, "pointer not aligned to its elements");
            const auto add = [&](const void* p, int64_t n, size_t bytes) { written.push_back(range_of(p, n, bytes)); };
            add(t.param, t.count, size);
            add(t.mean, t.count, state);
            add(t.square, t.count, state);
            if (t.copy) add(t.copy, t.count, type_bytes(copy_type));
            if (state_bits == 8) {
                add(t.mean_scale, ceil_div(t.count, P2_STATE_BLOCK), 4);
                add(t.square_scale, ceil_div(t.count, P2_STATE_BLOCK), 4);
            }
        }
        if (overlap(written)) return api_fail(P2_EINVAL, "tensors overlap");
        for (int64_t i = 0; i < n; ++i) {
            const p2_adamw_tensor& t = tensors[i];
            if (t.count > 0 && !(t.grad == t.copy && grad_type == copy_type) && overlap(written, range_of(t.grad, t.count, type_bytes(grad_type))))
                return api_fail(P2_EINVAL, "a gradient overlaps what is written");
        }
        if (!step || !aligned_to(step, 8) || !aligned_to(rate, 4) || !aligned_to(square_sum, 8)) return api_fail(P2_EINVAL, "step null, or pointer not aligned to its elements");
        if (!workspace || !aligned_to(workspace, 256)) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < 256) return api_fail(P2_ENOSPC, "workspace too small");
        const Range own[2] = {range_of(step, 1, 8), range_of(workspace, 256, 1)}, read[2] = {range_of(rate, rate ? 1 : 0, 4), range_of(square_sum, square_sum ? 1 : 0, 8)};
        const auto apart = [](const Range& x, const Range& y) { return x.second <= y.first || y.second <= x.first; };
        for (const Range& w : own)
            if (overlap(written, w) || !apart(w, read[0]) || !apart(w, read[1])) return api_fail(P2_EINVAL, "step or workspace overlaps what is written or read");
        if (!apart(own[0], own[1])) return api_fail(P2_EINVAL, "step and workspace overlap");
        for (const Range& r : read)
            if (r.first != r.second && overlap(written, r)) return api_fail(P2_EINVAL, "rate or square_sum overlaps what is written");
        for (int64_t i = 0; i < n; ++i)
            for (const Range& w : own)
                if (tensors[i].count > 0 && !apart(range_of(tensors[i].grad, tensors[i].count, type_bytes(grad_type)), w)) return api_fail(P2_EINVAL, "a gradient overlaps step or workspace");
        Adamw a = {};
        a.tensors = tensors; a.n = n; a.numbers = static_cast<AdamwStep*>(workspace); a.eps = eps;
        a.call = {step, rate, square_sum, lr, beta1, beta2, weight_decay, grad_factor, max_norm};
        a.type = type; a.grad_type = grad_type; a.copy_type = copy_type; a.state_bits = state_bits;
        return launched(launch_adamw(a, (hipStream_t)stream), "AdamW");
    });
}

int32_t p2_adamw_values(const p2_adamw_tensor* tensors, int64_t n, float* const* mean_out, float* const* square_out, void* stream) {
    return guarded([&]() -> int32_t {
        if (n > 0 && !tensors) return api_fail(P2_EINVAL, "null argument");
        int32_t rc = check_tensors(n, [&](int64_t i) { return tensors[i].count; });
        if (rc != P2_OK) return rc;
        for (int64_t i = 0; i < n; ++i) {
            const p2_adamw_tensor& t = tensors[i];
            const float *m = mean_out ? mean_out[i] : nullptr, *s = square_out ? square_out[i] : nullptr;
            if (t.count > 0 && ((m && (!t.mean || !t.mean_scale)) || (s && (!t.square || !t.square_scale)))) return api_fail(P2_EINVAL, "null argument");
            if (!aligned_to(m, 4) || !aligned_to(s, 4) || !aligned_to(t.mean_scale, 4) || !aligned_to(t.square_scale, 4))
                return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        }
        return launched(launch_adamw_values(tensors, n, mean_out, square_out, (hipStream_t)stream), "AdamW's values");
    });
}

int32_t p2_linear_forward_workspace(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, int32_t type, int64_t rows, int64_t inner,
                                    int64_t outer, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_linear(type, rows, inner, outer);
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        LinearForward a = {};
        a.x = x; a.x_stride = x_stride; a.weight = weight; a.weight_stride = weight_stride; a.type = type; a.rows = rows; a.inner = inner; a.outer = outer;
        *bytes = linear_forward_workspace(a);
        return P2_OK;
    });
}

int32_t p2_linear_forward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, const void* bias, const void* residual,
                          int64_t residual_stride, int32_t type, int32_t activation, int64_t rows, int64_t inner, int64_t outer, void* y, int64_t y_stride,
                          void* z, int64_t z_stride, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_linear(type, rows, inner, outer);
        if (rc != P2_OK) return rc;
        if (activation < P2_NO_ACTIVATION || activation > P2_SILU) return api_fail(P2_EINVAL, "unknown activation");
        for (const char* bad : {bad_rows(x, type, x_stride, rows, inner), bad_rows(weight, type, weight_stride, outer, inner), bad_rows(y, type, y_stride, rows, outer),
                                residual ? bad_rows(residual, type, residual_stride, rows, outer) : nullptr, z ? bad_rows(z, type, z_stride, rows, outer) : nullptr})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (!aligned_to(bias, type_bytes(type))) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        if (y && y == residual && rows > 1 && y_stride != residual_stride) return api_fail(P2_EINVAL, "y is residual with another stride");
        if (y && (y == x || y == z || y == weight)) return api_fail(P2_EINVAL, "y is an input, or z");
        if (z && (z == x || z == weight || z == residual)) return api_fail(P2_EINVAL, "z is an input");
        LinearForward a = {};
        a.x = x; a.weight = weight; a.bias = bias; a.residual = residual; a.y = y; a.z = z; a.workspace = static_cast<char*>(workspace);
        a.x_stride = x_stride; a.weight_stride = weight_stride; a.residual_stride = residual_stride; a.y_stride = y_stride; a.z_stride = z_stride;
        a.rows = rows; a.inner = inner; a.outer = outer; a.type = type; a.activation = activation;
        const int64_t room = linear_forward_workspace(a);
        if (room && (!workspace || !aligned_to(workspace, 256))) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < room) return api_fail(P2_ENOSPC, "workspace too small");
        if (rows == 0) return P2_OK;
        const Extent of_y = extent_of(y, type, y_stride, rows, outer), of_z = extent_of(z, type, z_stride, rows, outer), of_work = extent_of(room ? workspace : nullptr, P2_F32, 0, 1, room / 4);
        const Extent of_residual = extent_of(residual, type, residual_stride, rows, outer);
        const Extent read[] = {extent_of(x, type, x_stride, rows, inner), extent_of(weight, type, weight_stride, outer, inner), extent_of(bias, type, 0, 1, outer)};
        for (const Extent& r : read)
            if (overlap(of_y, r) || overlap(of_z, r) || overlap(of_work, r)) return api_fail(P2_EINVAL, "y, z or workspace overlaps an input");
        if ((y != residual && overlap(of_y, of_residual)) || overlap(of_z, of_residual) || overlap(of_work, of_residual)) return api_fail(P2_EINVAL, "y, z or workspace overlaps the residual");
        if (overlap(of_y, of_z) || overlap(of_y, of_work) || overlap(of_z, of_work)) return api_fail(P2_EINVAL, "y, z and workspace overlap");
        return launched(launch_linear_forward(a, (hipStream_t)stream), "linear");
    });
}

int32_t p2_linear_backward_workspace(int32_t type, int64_t rows, int64_t inner, int64_t outer, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_linear(type, rows, inner, outer);
        if (rc != P2_OK) return rc;
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        *bytes = linear_backward_workspace(type, rows, inner, outer);
        return P2_OK;
    });
}

int32_t p2_linear_backward_workspace_for(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, int32_t type,
                                         int32_t activation, int64_t rows, int64_t inner, int64_t outer, int32_t dx, int32_t dweight, int32_t dbias, int64_t* bytes) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_linear(type, rows, inner, outer);
        if (rc != P2_OK) return rc;
        if (activation < P2_NO_ACTIVATION || activation > P2_SILU) return api_fail(P2_EINVAL, "unknown activation");
        if (!bytes) return api_fail(P2_EINVAL, "null argument");
        LinearBackward a = {};
        a.dy = dy; a.dy_stride = dy_stride; a.x = x; a.x_stride = x_stride; a.weight = weight; a.weight_stride = weight_stride;
        a.dx = dx ? bytes : nullptr; a.dweight = dweight ? bytes : nullptr; a.dbias = dbias ? bytes : nullptr;         // (asked for or not)
        a.rows = rows; a.inner = inner; a.outer = outer; a.type = type; a.activation = activation;
        *bytes = linear_backward_workspace(a);
        return P2_OK;
    });
}

int32_t p2_linear_backward(const void* dy, int64_t dy_stride, const void* z, int64_t z_stride, const void* x, int64_t x_stride, const void* weight,
                           int64_t weight_stride, int32_t type, int32_t activation, int64_t rows, int64_t inner, int64_t outer, void* dx, int64_t dx_stride,
                           void* dweight, int64_t dweight_stride, void* dbias, int32_t weight_type, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&]() -> int32_t {
        int32_t rc = check_linear(type, rows, inner, outer);
        if (rc != P2_OK) return rc;
        if (!known_type(weight_type)) return api_fail(P2_EINVAL, "unknown element type");
        if (activation < P2_NO_ACTIVATION || activation > P2_SILU) return api_fail(P2_EINVAL, "unknown activation");
        const bool slope = activation != P2_NO_ACTIVATION;
        for (const char* bad : {bad_rows(dy, type, dy_stride, rows, outer), slope ? bad_rows(z, type, z_stride, rows, outer) : nullptr,
                                dweight ? bad_rows(x, type, x_stride, rows, inner) : nullptr, dx ? bad_rows(weight, type, weight_stride, outer, inner) : nullptr,
                                dx ? bad_rows(dx, type, dx_stride, rows, inner) : nullptr, dweight ? bad_rows(dweight, weight_type, dweight_stride, outer, inner) : nullptr})
            if (bad) return api_fail(P2_EINVAL, bad);
        if (!aligned_to(dbias, type_bytes(weight_type))) return api_fail(P2_EINVAL, "pointer not aligned to its elements");
        if (dx && (dx == dy || dx == x || dx == weight || dx == z || dx == dweight)) return api_fail(P2_EINVAL, "dx is an input, or dweight");
        if (dweight && (dweight == dy || dweight == x || dweight == weight || dweight == z)) return api_fail(P2_EINVAL, "dweight is an input");
        LinearBackward a = {};
        a.dy = dy; a.z = z; a.x = x; a.weight = weight; a.dx = dx; a.dweight = dweight; a.dbias = dbias; a.workspace = static_cast<char*>(workspace);
        a.dy_stride = dy_stride; a.z_stride = z_stride; a.x_stride = x_stride; a.weight_stride = weight_stride; a.dx_stride = dx_stride;
        a.dweight_stride = dweight_stride; a.rows = rows; a.inner = inner; a.outer = outer; a.type = type; a.activation = activation; a.weight_type = weight_type;
        const int64_t room = linear_backward_workspace(a);
        if (room && (!workspace || !aligned_to(workspace, 256))) return api_fail(P2_EINVAL, "workspace null or not aligned to 256");
        if (workspace_bytes < room) return api_fail(P2_ENOSPC, "workspace too small");
        const Extent written[] = {extent_of(dx, type, dx_stride, rows, inner), extent_of(dweight, weight_type, dweight_stride, outer, inner), extent_of(dbias, weight_type, 0, 1, outer),
                                  extent_of(room ? workspace : nullptr, P2_F32, 0, 1, room / 4)};
        const Extent read[] = {extent_of(dy, type, dy_stride, rows, outer), extent_of(slope ? z : nullptr, type, z_stride, rows, outer), extent_of(dweight ? x : nullptr, type, x_stride, rows, inner),
                               extent_of(dx ? weight : nullptr, type, weight_stride, outer, inner)};
        for (int i = 0; i < 4; ++i) {
            for (const Extent& r : read)
                if (overlap(written[i], r)) return api_fail(P2_EINVAL, "a gradient or workspace overlaps an input");
            for (int j = 0; j < i; ++j)
                if (overlap(written[i], written[j])) return api_fail(P2_EINVAL, "gradients or workspace overlap");
        }
        return launched(launch_linear_backward(a, (hipStream_t)stream), "linear's gradients");
    });
}

}  // extern "C"
