// Layer norm, forward and backward.
//
// A row is read once and stays in registers: its mean, the mean of its centred squares (no difference of large sums) and the
// result are worked out from there, so that a pass moves what it cannot do without: 2 values an element forward, 3 backward.
// Rows are dealt to groups of kTpr threads (a part of a wavefront, a wavefront, or a block), each thread holding kNv vectors
// of 16 bytes.
#include <algorithm>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kNormBlock = 256;            // threads of a block whose rows take less than a block
constexpr int64_t kMaxNormBlocks = 1 << 20;

template <int kTpr> struct NormGroup {
    static constexpr int kThreads = kTpr < kNormBlock ? kNormBlock : kTpr;
    static constexpr int kRows = kThreads / kTpr;
    static constexpr int kWaves = kTpr / 64;               // wavefronts of a row that has several
};

// Sum over the threads of a row.  `buf`: a float per wavefront, another one for each sum between two barriers.
template <int kTpr> __device__ __forceinline__ float row_sum(float v, float* buf) {
    if constexpr (kTpr <= 64) {
        return group_sum<kTpr>(v);
    } else {
        constexpr int kWaves = kTpr / 64;
        v = group_sum<64>(v);
        if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += buf[(threadIdx.x / kTpr) * kWaves + w];
        return s;
    }
}

// N weights from column c on, in whatever type they have; loaded like a row's vectors.
template <int N, bool kWhole> struct WeightVec {
    RowVec<float, N, kWhole> raw;              // 16-bit types: the first half of it
    __device__ __forceinline__ void load(const void* p, int32_t type, int c, int cols) {
        if (type == P2_F32) {
            raw.load(static_cast<const float*>(p), c, cols);
        } else {
            RowVec<half_t, N, kWhole> r;
            r.load(static_cast<const half_t*>(p), c, cols);
            typedef float part_t __attribute__((ext_vector_type(N / 2)));
            const part_t w = __builtin_bit_cast(part_t, r.raw);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) raw.raw[i] = w[i];
        }
    }
    template <typename T> __device__ __forceinline__ void get_narrow(int c, int cols, float other, float (&v)[N]) const {
        typedef float part_t __attribute__((ext_vector_type(N / 2)));
        part_t w;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = raw.raw[i];
        RowVec<T, N, kWhole> r;
        r.raw = __builtin_bit_cast(decltype(r.raw), w);
        r.get(c, cols, other, v);
    }
    __device__ __forceinline__ void get(int32_t type, int c, int cols, float other, float (&v)[N]) const {
        if (type == P2_F32) raw.get(c, cols, other, v);
        else if (type == P2_F16) get_narrow<half_t>(c, cols, other, v);
        else get_narrow<bf16_t>(c, cols, other, v);
    }
};

template <typename T, int kTpr, int kNv, bool kWhole> __global__ __launch_bounds__(NormGroup<kTpr>::kThreads) void k_norm_forward(NormForward a) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kRows = NormGroup<kTpr>::kRows;
    __shared__ float buf[2][16];
    const int lane = threadIdx.x % kTpr, cols = (int)a.cols;
    const float n = (float)a.cols;                         // (a row of equal values has exactly that mean: no product with 1 / n)
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (int64_t)gridDim.x * kRows) {
        const int64_t row = row0 + threadIdx.x / kTpr;
        const bool there = row < a.rows;                   // (rows of a block's own threads: all of them, or none)
        const T* x = static_cast<const T*>(a.x) + (there ? row : a.rows - 1) * a.x_stride;
        RowVec<T, V, kWhole> raw[kNv];
        WeightVec<V, kWhole> w[kNv], b[kNv];
#pragma unroll
        for (int i = 0; i < kNv; ++i) raw[i].load(x, (i * kTpr + lane) * V, cols);
        auto ask_weights = [&] {
            if (a.weight)
#pragma unroll
                for (int i = 0; i < kNv; ++i) w[i].load(a.weight, a.weight_type, (i * kTpr + lane) * V, cols);
            if (a.bias)
#pragma unroll
                for (int i = 0; i < kNv; ++i) b[i].load(a.bias, a.weight_type, (i * kTpr + lane) * V, cols);
        };
        if constexpr (kNv <= 2) ask_weights();             // (there are registers to have them wait in)
        float v[kNv][V];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
            raw[i].get((i * kTpr + lane) * V, cols, 0.0f, v[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) s += v[i][j];
        }
        const float mean = row_sum<kTpr>(s, buf[0]) / n;
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < kNv; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = (i * kTpr + lane) * V + (kWhole ? 0 : j);
                v[i][j] -= mean;
                s += c < cols ? v[i][j] * v[i][j] : 0.0f;
            }
        const float rstd = 1.0f / sqrtf(row_sum<kTpr>(s, buf[1]) / n + a.eps);
        if (there) {
            if constexpr (kNv > 2) ask_weights();
            if (lane == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
            T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int i = 0; i < kNv; ++i) {
                const int c = (i * kTpr + lane) * V;
                float wv[V], bv[V];
#pragma unroll
                for (int j = 0; j < V; ++j) { wv[j] = 1.0f; bv[j] = 0.0f; }
                if (a.weight) w[i].get(a.weight_type, c, cols, 1.0f, wv);
                if (a.bias) b[i].get(a.weight_type, c, cols, 0.0f, bv);
#pragma unroll
                for (int j = 0; j < V; ++j) wv[j] = v[i][j] * rstd * wv[j] + bv[j];
                if constexpr (kWhole) { if (c < cols) store_vec<T, V>(y + c, wv); }
                else store_part<T, V>(y + c, cols - c, wv);
            }
        }
    }
}

// Rows too long for registers, or shorter than a vector: three passes over them, the later two from the cache.
template <typename T> __global__ __launch_bounds__(1024) void k_norm_forward_long(NormForward a) {
    __shared__ float buf[2][16];
    const float n = (float)a.cols;                         // (a row of equal values has exactly that mean: no product with 1 / n)
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        float s = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += 1024) s += (float)x[c];
        const float mean = row_sum<1024>(s, buf[0]) / n;
        s = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += 1024) { const float d = (float)x[c] - mean; s += d * d; }
        const float rstd = 1.0f / sqrtf(row_sum<1024>(s, buf[1]) / n + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        T* y = static_cast<T*>(a.y) + row * a.y_stride;
        for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
            float w[1] = {1.0f}, b[1] = {0.0f};
            if (a.weight) load_typed<1>(a.weight, a.weight_type, c, 1, w, 1.0f);
            if (a.bias) load_typed<1>(a.bias, a.weight_type, c, 1, b, 0.0f);
            y[c] = (T)(((float)x[c] - mean) * rstd * w[0] + b[0]);
        }
    }
}

// Backward.  A block takes every gridDim.x-th group of rows and keeps its columns' sums of dy * xh and dy in registers
// the whole time; at its end they are added up over the block's row groups in a fixed order and written as one line of
// partial sums, which k_norm_weight_grad adds up.
constexpr int kBackBlock = 512;
constexpr int64_t kBackBlocks = 512;       // two blocks a compute unit: 16 wavefronts

template <typename T, int kTpr, int kNv, bool kWhole> __global__ __launch_bounds__(kBackBlock) void k_norm_backward(NormBackward a) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kRows = kBackBlock / kTpr;
    constexpr int kCols = kTpr * kNv * V;
    __shared__ float buf[2][2][kBackBlock / 64];
    __shared__ float sums[2][kRows > 1 ? kCols : 1];
    const int lane = threadIdx.x % kTpr, group = threadIdx.x / kTpr, cols = (int)a.cols;
    const float inv = 1.0f / (float)a.cols;
    float w[kNv][V], dw[kNv][V], db[kNv][V];
#pragma unroll
    for (int i = 0; i < kNv; ++i) {
        const int c = (i * kTpr + lane) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) { w[i][j] = 1.0f; dw[i][j] = 0.0f; db[i][j] = 0.0f; }
        if (a.weight) load_typed<V>(a.weight, a.weight_type, c, cols - c, w[i], 0.0f);
    }
    // A row's values are asked for while the row before it is worked on.
    RowVec<T, V, kWhole> nx[kNv], nd[kNv];
    float next_mean, next_rstd;
    auto ask = [&](int64_t row) {
        const int64_t at = row < a.rows ? row : a.rows - 1;
        const T* x = static_cast<const T*>(a.x) + at * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + at * a.dy_stride;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
            nx[i].load(x, (i * kTpr + lane) * V, cols);
            nd[i].load(dy, (i * kTpr + lane) * V, cols);
        }
        next_mean = a.mean[at];
        next_rstd = a.rstd[at];
    };
    const int64_t stride = (int64_t)gridDim.x * kRows;
    int turn = 0;
    constexpr bool kEarly = kNv <= 2;                      // (more vectors would not stay in registers)
    if constexpr (kEarly) ask((int64_t)blockIdx.x * kRows + group);
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += stride, turn ^= 1) {
        const int64_t row = row0 + group;
        const bool there = row < a.rows;
        if constexpr (!kEarly) ask(row);
        const float mean = next_mean, rstd = next_rstd;
        float xh[kNv][V], d[kNv][V];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
            const int c = (i * kTpr + lane) * V;
            nx[i].get(c, cols, mean, xh[i]);
            nd[i].get(c, cols, 0.0f, d[i]);
        }
        if constexpr (kEarly) { if (row0 + stride < a.rows) ask(row + stride); }
#pragma unroll
        for (int i = 0; i < kNv; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                xh[i][j] = (xh[i][j] - mean) * rstd;
                const float t = d[i][j] * xh[i][j];
                dw[i][j] += there ? t : 0.0f;
                db[i][j] += there ? d[i][j] : 0.0f;
                d[i][j] *= w[i][j];
                s1 += d[i][j];
                s2 += t * w[i][j];
            }
        if (a.dx) {
            // two sums at one barrier; the buffers of the next row are other ones
            float m1, m2;
            if constexpr (kTpr <= 64) {
                m1 = group_sum<kTpr>(s1) * inv;
                m2 = group_sum<kTpr>(s2) * inv;
            } else {
                s1 = group_sum<64>(s1);
                s2 = group_sum<64>(s2);
                if ((threadIdx.x & 63) == 0) { buf[turn][0][threadIdx.x >> 6] = s1; buf[turn][1][threadIdx.x >> 6] = s2; }
                __syncthreads();
                m1 = m2 = 0.0f;
#pragma unroll
                for (int q = 0; q < kTpr / 64; ++q) { m1 += buf[turn][0][group * (kTpr / 64) + q]; m2 += buf[turn][1][group * (kTpr / 64) + q]; }
                m1 *= inv;
                m2 *= inv;
            }
            if (there) {
                T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
#pragma unroll
                for (int i = 0; i < kNv; ++i) {
                    const int c = (i * kTpr + lane) * V;
                    float o[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) o[j] = rstd * (d[i][j] - m1 - xh[i][j] * m2);
                    if constexpr (kWhole) { if (c < cols) store_vec<T, V>(dx + c, o); }
                    else store_part<T, V>(dx + c, cols - c, o);
                }
            }
        }
    }
    if (!a.partial) return;
    float* line = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
            const int64_t c = (int64_t)(i * kTpr + lane) * V;
            store_part<float, V>(line + c, a.cols - c, dw[i]);
            store_part<float, V>(line + a.cols + c, a.cols - c, db[i]);
        }
    } else {
        for (int g = 0; g < kRows; ++g) {
            if (group == g) {
#pragma unroll
                for (int i = 0; i < kNv; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int c = (i * kTpr + lane) * V + j;
                        sums[0][c] = g ? sums[0][c] + dw[i][j] : dw[i][j];
                        sums[1][c] = g ? sums[1][c] + db[i][j] : db[i][j];
                    }
            }
            __syncthreads();
        }
        for (int64_t c = threadIdx.x; c < a.cols; c += kBackBlock) {
            line[c] = sums[0][c];
            line[a.cols + c] = sums[1][c];
        }
    }
}

template <typename T> __global__ __launch_bounds__(1024) void k_norm_backward_long(NormBackward a) {
    __shared__ float buf[2][16];
    const float inv = 1.0f / (float)a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
            float w[1] = {1.0f};
            if (a.weight) load_typed<1>(a.weight, a.weight_type, c, 1, w, 1.0f);
            const float g = (float)dy[c] * w[0];
            s1 += g;
            s2 += g * (((float)x[c] - mean) * rstd);
        }
        const float m1 = row_sum<1024>(s1, buf[0]) * inv;
        const float m2 = row_sum<1024>(s2, buf[1]) * inv;
        T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
        for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
            float w[1] = {1.0f};
            if (a.weight) load_typed<1>(a.weight, a.weight_type, c, 1, w, 1.0f);
            dx[c] = (T)(rstd * ((float)dy[c] * w[0] - m1 - ((float)x[c] - mean) * rstd * m2));
        }
    }
}

// Partial sums of rows too long for registers: a block takes 256 columns of every gridDim.y-th row.
template <typename T> __global__ __launch_bounds__(256) void k_norm_columns_long(NormBackward a) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float d = (float)static_cast<const T*>(a.dy)[row * a.dy_stride + c];
        dw += d * (((float)static_cast<const T*>(a.x)[row * a.x_stride + c] - a.mean[row]) * a.rstd[row]);
        db += d;
    }
    float* line = a.partial + (int64_t)blockIdx.y * 2 * a.cols;
    line[c] = dw;
    line[a.cols + c] = db;
}

// dweight (blockIdx.y = 0) and dbias (1) from `lines` lines of partial sums: 16 columns a block, 64 threads a column.
__global__ __launch_bounds__(1024) void k_norm_weight_grad(const float* __restrict__ partial, int64_t lines, int64_t cols, void* dweight,
                                                           void* dbias, int32_t weight_type) {
    __shared__ float part[64][17];
    void* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int x = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + x;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int64_t l = r; l < lines; l += 64) s += partial[(l * 2 + blockIdx.y) * cols + c];
    part[r][x] = s;
    for (int d = 32; d >= 1; d >>= 1) {
        __syncthreads();
        if (r < d) part[r][x] += part[r + d][x];
    }
    if (r == 0 && c < cols) store_typed(out, weight_type, c, part[0][x]);
}

template <typename T, int kTpr, int kNv> void forward_as(const NormForward& a, hipStream_t s) {
    constexpr int kRows = NormGroup<kTpr>::kRows;
    const dim3 grid((unsigned)std::min(ceil_div(a.rows, kRows), kMaxNormBlocks)), block(NormGroup<kTpr>::kThreads);
    if (a.cols % (16 / sizeof(T)) == 0) k_norm_forward<T, kTpr, kNv, true><<<grid, block, 0, s>>>(a);
    else k_norm_forward<T, kTpr, kNv, false><<<grid, block, 0, s>>>(a);
}

template <typename T> void forward_of(const NormForward& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int64_t vecs = ceil_div(a.cols, V);
    if (a.cols < V || vecs > 4096) k_norm_forward_long<T><<<dim3((unsigned)std::min(a.rows, kMaxNormBlocks)), dim3(1024), 0, s>>>(a);
    else if (vecs <= 16) forward_as<T, 16, 1>(a, s);
    else if (vecs <= 64) forward_as<T, 64, 1>(a, s);
    else if (vecs <= 128) forward_as<T, 64, 2>(a, s);
    else if (vecs <= 256) forward_as<T, 256, 1>(a, s);
    else if (vecs <= 512) forward_as<T, 256, 2>(a, s);
    else if (vecs <= 1024) forward_as<T, 256, 4>(a, s);
    else forward_as<T, 1024, 4>(a, s);
}

// Threads and vectors of a row in the backward pass; 0: too long for registers.
struct BackShape { int tpr, nv; };
BackShape back_shape(int64_t cols, int64_t v) {
    const int64_t vecs = ceil_div(cols, v);
    if (cols < v) return {0, 0};
    if (vecs <= 16) return {16, 1};
    if (vecs <= 64) return {64, 1};
    if (vecs <= 128) return {64, 2};
    if (vecs <= 256) return {256, 1};
    if (vecs <= 512) return {256, 2};
    if (vecs <= 1024) return {512, 2};
    if (vecs <= 2048) return {512, 4};
    return {0, 0};
}

template <typename T, int kTpr, int kNv> void backward_as(const NormBackward& a, int64_t blocks, hipStream_t s) {
    if (a.cols % (16 / sizeof(T)) == 0) k_norm_backward<T, kTpr, kNv, true><<<dim3((unsigned)blocks), dim3(kBackBlock), 0, s>>>(a);
    else k_norm_backward<T, kTpr, kNv, false><<<dim3((unsigned)blocks), dim3(kBackBlock), 0, s>>>(a);
}

int64_t back_blocks(int64_t rows, int64_t cols, int32_t value_bytes) {
    const BackShape f = back_shape(cols, 16 / value_bytes);
    const int64_t groups = f.tpr ? ceil_div(rows, kBackBlock / f.tpr) : rows;
    return std::max<int64_t>(1, std::min(groups, kBackBlocks));
}

template <typename T> hipError_t backward_of(const NormBackward& a, hipStream_t s) {
    const BackShape f = back_shape(a.cols, 16 / (int64_t)sizeof(T));
    const int64_t blocks = back_blocks(a.rows, a.cols, sizeof(T));
    if (a.rows > 0) {
        switch (f.tpr * 8 + f.nv) {
            case 16 * 8 + 1: backward_as<T, 16, 1>(a, blocks, s); break;
            case 64 * 8 + 1: backward_as<T, 64, 1>(a, blocks, s); break;
            case 64 * 8 + 2: backward_as<T, 64, 2>(a, blocks, s); break;
            case 256 * 8 + 1: backward_as<T, 256, 1>(a, blocks, s); break;
            case 256 * 8 + 2: backward_as<T, 256, 2>(a, blocks, s); break;
            case 512 * 8 + 2: backward_as<T, 512, 2>(a, blocks, s); break;
            case 512 * 8 + 4: backward_as<T, 512, 4>(a, blocks, s); break;
            default:
                // (the columns first: dx may be dy)
                if (a.partial) k_norm_columns_long<T><<<dim3((unsigned)ceil_div(a.cols, 256), (unsigned)blocks), dim3(256), 0, s>>>(a);
                if (a.dx) k_norm_backward_long<T><<<dim3((unsigned)std::min(a.rows, kMaxNormBlocks)), dim3(1024), 0, s>>>(a);
        }
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.partial)
        k_norm_weight_grad<<<dim3((unsigned)ceil_div(a.cols, 16), 2), dim3(1024), 0, s>>>(a.partial, a.rows > 0 ? blocks : 0, a.cols, a.dweight, a.dbias, a.weight_type);
    return hipGetLastError();
}

}  // namespace

int64_t norm_backward_partials(int64_t rows, int64_t cols) {
    return std::max(back_blocks(rows, cols, 2), back_blocks(rows, cols, 4)) * 2 * cols;
}

hipError_t launch_norm_forward(const NormForward& a, hipStream_t s) {
    if (a.type == P2_F32) forward_of<float>(a, s);
    else if (a.type == P2_BF16) forward_of<bf16_t>(a, s);
    else forward_of<half_t>(a, s);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormBackward& a, hipStream_t s) {
    if (a.type == P2_F32) return backward_of<float>(a, s);
    if (a.type == P2_BF16) return backward_of<bf16_t>(a, s);
    return backward_of<half_t>(a, s);
}

}  // namespace p2
