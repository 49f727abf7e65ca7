// Layer norm, forward and backward.
//
// A row is read once and stays in registers: its mean, with what the first sum of it rounded off, the mean of its centred squares and
// the result are worked out from there, so that a pass moves what it cannot do without: 2 values an element forward, 3 backward.
// Rows are dealt to groups of kTpr threads (a part of a wavefront, a wavefront, or a block), each thread holding kNv vectors
// of 16 bytes.
//
// What bounds it: memory.  A copy of 4 GiB reaches 4.84 TB/s here; forward, 8192 x 4096 bf16: 25.9 us, 5.2 TB/s (part of it from the last
// cache; 24 without what the first mean rounds off, which a row of 5000 fp32 values of 12345.678 pays for with results of 0.5 for 0); backward with both sums,
// 16384 x 4096 bf16: 80.9 us, 5.0 TB/s, of which k_norm_weight_grad takes 4.9.  Rows with odd ends: 5003 x 1023 fp16 of rows 1061 apart 8 us, 2.6 TB/s.  One
// row: 2.4 us on the device in a call of 6.7.
#include <algorithm>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kNormBlock = 256;            // threads of a block whose rows take less than a block
constexpr int64_t kMaxNormBlocks = 1 << 20;
constexpr int64_t kForwardThreads = 256 * 2048;          // rows beyond what fills the chip are dealt out in turn

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

// Two of them at one barrier.
template <int kTpr> __device__ __forceinline__ void row_sums(float& a, float& b, float* buf_a, float* buf_b) {
    if constexpr (kTpr <= 64) {
        a = group_sum<kTpr>(a);
        b = group_sum<kTpr>(b);
    } else {
        constexpr int kWaves = kTpr / 64;
        a = group_sum<64>(a);
        b = group_sum<64>(b);
        if ((threadIdx.x & 63) == 0) { buf_a[threadIdx.x >> 6] = a; buf_b[threadIdx.x >> 6] = b; }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) { a += buf_a[(threadIdx.x / kTpr) * kWaves + w]; b += buf_b[(threadIdx.x / kTpr) * kWaves + w]; }
    }
}

// What a row's first mean rounded off, and its spread.  A sum of n values in 32 bits rounds, so the first mean is off by some steps of its own
// size, which may be more than the whole spread of a row that lies far from zero.  What the values' distances from it sum up to is taken off again:
// the mean is mean + low, a centred value (x - mean) - low, the variance that of those.  It comes from the distances' squares, less low^2, as long as
// that loses a bit at most, which two sums at one barrier suffice for; else (rows of equal values, nearly) the rest is taken off, too, and the squares
// are summed afresh.
// each(f): f(x - mean, whether it counts) for this thread's values.  kTpr: threads of the row, which are a block's where it has several wavefronts
// (the barriers); buf: a line for each sum, the first of which is the mean's, so that the next row's is written when all have read this one's.
struct Centre {
    float low, rstd;
    __device__ __forceinline__ float of(float d) const { return (d - low) * rstd; }
    __device__ __forceinline__ float whole_mean(float mean) const { return low == low ? mean + low : mean; }     // (an infinity beside numbers has an infinite mean)
};
constexpr int kSumLines = 5;
template <int kTpr, typename Each> __device__ __forceinline__ Centre centre_of(float n, float eps, float (*buf)[16], Each&& each) {
    float s = 0.0f, q = 0.0f;
    each([&](float d, bool counts) { const float v = counts ? d : 0.0f; s += v; q += v * v; });
    row_sums<kTpr>(s, q, buf[1], buf[2]);
    Centre c;
    c.low = s / n;
    const float square = c.low * c.low;
    float variance = q / n - square;
    if (!(variance >= square && square < INFINITY)) {      // (the same for all threads of the row)
        s = q = 0.0f;
        each([&](float d, bool counts) { s += counts ? d - c.low : 0.0f; });
        c.low += row_sum<kTpr>(s, buf[3]) / n;
        each([&](float d, bool counts) { const float v = counts ? d - c.low : 0.0f; q += v * v; });
        variance = row_sum<kTpr>(q, buf[4]) / n;
    }
    c.rstd = 1.0f / sqrtf(variance + eps);
    return c;
}

// A lane's N weights, in whatever type they have; loaded like a row's vectors.
template <int N> struct WeightVec {
    vec_t<float, N> raw;                       // 16-bit types: the first half of it
    __device__ __forceinline__ void load(const void* p, int32_t type, int c, int cols) {
        if (type == P2_F32) {
            raw = load_whole<float, N>(static_cast<const float*>(p), c, cols);
        } else {
            typedef float part_t __attribute__((ext_vector_type(N / 2)));
            const part_t w = __builtin_bit_cast(part_t, load_whole<half_t, N>(static_cast<const half_t*>(p), c, cols));
#pragma unroll
            for (int i = 0; i < N / 2; ++i) raw[i] = w[i];
        }
    }
    __device__ __forceinline__ void get(int32_t type, float (&v)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (type == P2_F32) {
                v[i] = raw[i];
            } else {
                const uint32_t w = __float_as_uint(raw[i / 2]);
                const uint16_t h = (uint16_t)(i % 2 ? w >> 16 : w);
                v[i] = type == P2_BF16 ? __uint_as_float((uint32_t)h << 16) : (float)__builtin_bit_cast(half_t, h);
            }
        }
    }
};

// mean = sum x / n, rstd = 1 / sqrt(sum (x - mean)^2 / n + eps), y = (x - mean) rstd w + b.
template <typename T, int kTpr, int kNv, bool kWhole> __global__ __launch_bounds__(NormGroup<kTpr>::kThreads) void k_norm_forward(NormForward a) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kRows = NormGroup<kTpr>::kRows;
    constexpr bool kEarly = kNv <= 2;                      // weights for all rows, and a row ahead, stay in registers
    static_assert(kTpr <= 64 || kRows == 1, "rows of several wavefronts have a block each");
    __shared__ float buf[kSumLines][16];
    const int lane = threadIdx.x % kTpr, group = threadIdx.x / kTpr, cols = (int)a.cols;
    vec_t<T, V> next[kNv];
    auto ask = [&](int64_t row) {                          // (rows of a block's own threads: all of them are there, or none)
        const T* x = static_cast<const T*>(a.x) + (row < a.rows ? row : a.rows - 1) * a.x_stride;
#pragma unroll
        for (int i = 0; i < kNv; ++i) next[i] = load_whole<T, V>(x, (i * kTpr + lane) * V, cols);
    };
    WeightVec<V> raw_w[kNv], raw_b[kNv];
    auto ask_weights = [&] {
        if (a.weight)
#pragma unroll
            for (int i = 0; i < kNv; ++i) raw_w[i].load(a.weight, a.weight_type, (i * kTpr + lane) * V, cols);
        if (a.bias)
#pragma unroll
            for (int i = 0; i < kNv; ++i) raw_b[i].load(a.bias, a.weight_type, (i * kTpr + lane) * V, cols);
    };
    float w[kEarly ? kNv : 1][V], b[kEarly ? kNv : 1][V];
    auto weights_of = [&](int i, float (&wv)[V], float (&bv)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) { wv[j] = 1.0f; bv[j] = 0.0f; }
        if (a.weight) raw_w[i].get(a.weight_type, wv);
        if (a.bias) raw_b[i].get(a.weight_type, bv);
    };
    const int64_t stride = (int64_t)gridDim.x * kRows;
    if constexpr (kEarly) {
        ask((int64_t)blockIdx.x * kRows + group);
        ask_weights();
#pragma unroll
        for (int i = 0; i < kNv; ++i) weights_of(i, w[i], b[i]);
    }
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += stride) {
        const int64_t row = row0 + group;
        const bool there = row < a.rows;
        if constexpr (!kEarly) ask(row);
        float v[kNv][V];
        auto each = [&](auto&& f) {
#pragma unroll
            for (int i = 0; i < kNv; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) f(v[i][j], own<V, kWhole>((i * kTpr + lane) * V, cols, j));
        };
#pragma unroll
        for (int i = 0; i < kNv; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = (float)next[i][j];
        if constexpr (kEarly) { if (row0 + stride < a.rows) ask(row + stride); }
        float s = 0.0f;
        each([&](float x, bool counts) { s += counts ? x : 0.0f; });
        const float n = (float)a.cols, mean = row_sum<kTpr>(s, buf[0]) / n;
        each([&](float& x, bool) { x -= mean; });
        const Centre c = centre_of<kTpr>(n, a.eps, buf, each);
        if (there) {
            if constexpr (!kEarly) ask_weights();
            if (lane == 0) {
                if (a.mean) a.mean[row] = c.whole_mean(mean);
                if (a.rstd) a.rstd[row] = c.rstd;
            }
            T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int i = 0; i < kNv; ++i) {
                const int at = (i * kTpr + lane) * V;
                if constexpr (!kEarly) weights_of(i, w[0], b[0]);
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = c.of(v[i][j]) * w[kEarly ? i : 0][j] + b[kEarly ? i : 0][j];
                if (at < cols) store_vec<T, V>(y + vec_at(at, cols, V), o);
            }
        }
    }
}

// Rows too long for registers (more than 4096 vectors): three passes over them (five where the mean is taken off once more), the later ones from the cache.
template <typename T> __global__ __launch_bounds__(1024) void k_norm_forward_long(NormForward a) {
    __shared__ float buf[kSumLines][16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        float s = 0.0f;
        for (int64_t i = threadIdx.x; i < a.cols; i += 1024) s += (float)x[i];
        const float n = (float)a.cols, mean = row_sum<1024>(s, buf[0]) / n;
        const Centre c = centre_of<1024>(n, a.eps, buf, [&](auto&& f) {
            for (int64_t i = threadIdx.x; i < a.cols; i += 1024) f((float)x[i] - mean, true);
        });
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = c.whole_mean(mean);
            if (a.rstd) a.rstd[row] = c.rstd;
        }
        T* y = static_cast<T*>(a.y) + row * a.y_stride;
        for (int64_t i = threadIdx.x; i < a.cols; i += 1024) {
            float w[1] = {1.0f}, b[1] = {0.0f};
            if (a.weight) load_typed<1>(a.weight, a.weight_type, i, 1, w, 1.0f);
            if (a.bias) load_typed<1>(a.bias, a.weight_type, i, 1, b, 0.0f);
            y[i] = (T)(c.of((float)x[i] - mean) * w[0] + b[0]);
        }
    }
}

// Rows shorter than a vector (three fp32 values, seven 16-bit ones): a thread each.
constexpr int kShortBlock = 256;
template <typename T> __global__ __launch_bounds__(kShortBlock) void k_norm_forward_short(NormForward a) {
    constexpr int kMost = 16 / sizeof(T) - 1;
    const int cols = (int)a.cols;
    for (int64_t row = (int64_t)blockIdx.x * kShortBlock + threadIdx.x; row < a.rows; row += (int64_t)gridDim.x * kShortBlock) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        T* y = static_cast<T*>(a.y) + row * a.y_stride;
        float v[kMost], s = 0.0f;
#pragma unroll
        for (int i = 0; i < kMost; ++i) { v[i] = i < cols ? (float)x[i] : 0.0f; s += v[i]; }
        const float n = (float)a.cols, mean = s / n;
#pragma unroll
        for (int i = 0; i < kMost; ++i) v[i] -= mean;
        const Centre c = centre_of<1>(n, a.eps, nullptr, [&](auto&& f) {
#pragma unroll
            for (int i = 0; i < kMost; ++i) f(v[i], i < cols);
        });
        if (a.mean) a.mean[row] = c.whole_mean(mean);
        if (a.rstd) a.rstd[row] = c.rstd;
#pragma unroll
        for (int i = 0; i < kMost; ++i)
            if (i < cols) {
                float w[1] = {1.0f}, b[1] = {0.0f};
                if (a.weight) load_typed<1>(a.weight, a.weight_type, i, 1, w, 1.0f);
                if (a.bias) load_typed<1>(a.bias, a.weight_type, i, 1, b, 0.0f);
                y[i] = (T)(c.of(v[i]) * w[0] + b[0]);
            }
    }
}

// Backward.  xh = (x - mean) rstd, g = dy w, dx = rstd (g - mean(g) - xh mean(g xh)).  A block takes every gridDim.x-th group of
// rows and keeps its columns' sums of dy * xh and dy in registers the whole time; at its end they are added up over the block's
// row groups in a fixed order and written as one line of partial sums, which k_norm_weight_grad adds up.  Two blocks of 512 threads a
// compute unit: in one of 1024, which would halve the lines, four rows wait for each other's barriers (16384 x 4096 231 us for 84).
constexpr int kBackBlock = 512;
constexpr int64_t kBackBlocks = 512;       // two blocks a compute unit: 16 wavefronts

template <typename T, int kTpr, int kNv, bool kWhole> __global__ __launch_bounds__(kBackBlock) void k_norm_backward(NormBackward a) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kRows = kBackBlock / kTpr;
    constexpr int kCols = kTpr * kNv * V;
    __shared__ float buf[2][2][kBackBlock / 64];
    constexpr int kPart = kTpr < 64 ? 64 : kTpr;           // threads whose sums are added up before they go to LDS
    __shared__ __attribute__((aligned(16))) float sums[kBackBlock / kPart][kRows > 1 ? kCols : 4];
    const int lane = threadIdx.x % kTpr, group = threadIdx.x / kTpr, cols = (int)a.cols;
    const float inv = 1.0f / (float)a.cols;
    float w[kNv][V], dw[kNv][V], db[kNv][V];
#pragma unroll
    for (int i = 0; i < kNv; ++i) {
        const int c = (i * kTpr + lane) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) { w[i][j] = 1.0f; dw[i][j] = 0.0f; db[i][j] = 0.0f; }
        if (a.weight) {
            WeightVec<V> raw;
            raw.load(a.weight, a.weight_type, c, cols);
            raw.get(a.weight_type, w[i]);
        }
    }
    // A row's values are asked for while the row before it is worked on.
    vec_t<T, V> nx[kNv], nd[kNv];
    float next_mean, next_rstd;
    auto ask = [&](int64_t row) {
        const int64_t at = row < a.rows ? row : a.rows - 1;
        const T* x = static_cast<const T*>(a.x) + at * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + at * a.dy_stride;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
            nx[i] = load_whole<T, V>(x, (i * kTpr + lane) * V, cols);
            nd[i] = load_whole<T, V>(dy, (i * kTpr + lane) * V, cols);
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
#pragma unroll
            for (int j = 0; j < V; ++j) {
                xh[i][j] = (float)nx[i][j];
                d[i][j] = (float)nd[i][j];
            }
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
                const bool mine = own<V, kWhole>((i * kTpr + lane) * V, cols, j);
                s1 += mine ? d[i][j] : 0.0f;
                s2 += mine ? t * w[i][j] : 0.0f;
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
                    if (c < cols) store_vec<T, V>(dx + vec_at(c, cols, V), o);
                }
            }
        }
    }
    if (!a.partial) return;
    float* line = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
            const int c = (i * kTpr + lane) * V, at = vec_at(c, cols, V);
            if (c < cols) {                                // (both lanes of a column have seen the same rows: the same sums)
                store_vec<float, V>(line + at, dw[i]);
                store_vec<float, V>(line + a.cols + at, db[i]);
            }
        }
    } else {
        // Groups of one wavefront first, then the wavefronts', side by side in LDS: a lane's values where its vectors would lie, so
        // that column c of the vector that the row's end cuts is found further right.
        const int cut = kWhole ? cols : (cols - 1) / V * V, further = cut - (cols - V);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int i = 0; i < kNv; ++i) {
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v[j] = which ? db[i][j] : dw[i][j];
#pragma unroll
                    for (int d = kTpr; d < 64; d <<= 1) v[j] += __shfl_xor(v[j], d, 64);
                }
                if (kTpr >= 64 || (threadIdx.x & 63) < kTpr) store_vec<float, V>(&sums[threadIdx.x / kPart][(i * kTpr + lane) * V], v);
            }
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += kBackBlock) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < kBackBlock / kPart; ++q) s += sums[q][kWhole || c < cut ? c : c + further];
                line[which * a.cols + c] = s;
            }
            __syncthreads();
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

// Rows shorter than a vector: dx, and a line of partial sums a block.
template <typename T> __global__ __launch_bounds__(kShortBlock) void k_norm_backward_short(NormBackward a) {
    constexpr int kMost = 16 / sizeof(T) - 1, kWaves = kShortBlock / 64;
    __shared__ float sums[kWaves][2][kMost];
    const int cols = (int)a.cols;
    const float inv = 1.0f / (float)a.cols;
    float w[kMost], dw[kMost], db[kMost];
#pragma unroll
    for (int c = 0; c < kMost; ++c) {
        float v[1] = {1.0f};
        if (a.weight && c < cols) load_typed<1>(a.weight, a.weight_type, c, 1, v, 1.0f);
        w[c] = v[0];
        dw[c] = db[c] = 0.0f;
    }
    for (int64_t row = (int64_t)blockIdx.x * kShortBlock + threadIdx.x; row < a.rows; row += (int64_t)gridDim.x * kShortBlock) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float xh[kMost], d[kMost], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int c = 0; c < kMost; ++c) {
            xh[c] = c < cols ? ((float)x[c] - mean) * rstd : 0.0f;
            d[c] = c < cols ? (float)dy[c] : 0.0f;
            const float t = d[c] * xh[c];
            dw[c] += t;
            db[c] += d[c];
            d[c] *= w[c];
            s1 += d[c];
            s2 += t * w[c];
        }
        s1 *= inv;
        s2 *= inv;
        if (a.dx) {
            T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
#pragma unroll
            for (int c = 0; c < kMost; ++c) if (c < cols) dx[c] = (T)(rstd * (d[c] - s1 - xh[c] * s2));
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int c = 0; c < kMost; ++c) {
        const float p = group_sum<64>(dw[c]), q = group_sum<64>(db[c]);
        if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6][0][c] = p; sums[threadIdx.x >> 6][1][c] = q; }
    }
    __syncthreads();
    if ((int)threadIdx.x < 2 * cols) {
        const int which = (int)threadIdx.x / cols, c = (int)threadIdx.x % cols;
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) s += sums[q][which][c];
        a.partial[((int64_t)blockIdx.x * 2 + which) * a.cols + c] = s;
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

// dweight (blockIdx.y = 0) and dbias (1) from `lines` lines of partial sums: 32 columns a block, whole lines of the cache (16 columns: every
// line fetched twice, 84.4 us for 81.6 a call with 16384 x 4096), 32 threads a column.  Sums of a wavefront's threads by lane exchange, then of the
// wavefronts in their order.
constexpr int kSumColumns = 32;
__global__ __launch_bounds__(1024) void k_norm_weight_grad(const float* __restrict__ partial, int64_t lines, int64_t cols, void* dweight,
                                                           void* dbias, int32_t weight_type) {
    constexpr int kWide = kSumColumns, kDeep = 1024 / kWide;
    __shared__ float part[16][kWide];
    void* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int x = threadIdx.x % kWide, r = threadIdx.x / kWide;
    const int64_t c = (int64_t)blockIdx.x * kWide + x;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int64_t l = r; l < lines; l += kDeep) s += partial[(l * 2 + blockIdx.y) * cols + c];
#pragma unroll
    for (int d = kWide; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) < kWide) part[threadIdx.x >> 6][x] = s;
    __syncthreads();
    if (r > 0 || c >= cols) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += part[w][x];
    store_typed(out, weight_type, c, s);
}

template <typename T, int kTpr, int kNv> void forward_as(const NormForward& a, hipStream_t s) {
    constexpr int kRows = NormGroup<kTpr>::kRows;
    const dim3 grid((unsigned)std::min(ceil_div(a.rows, kRows), kForwardThreads / NormGroup<kTpr>::kThreads)), block(NormGroup<kTpr>::kThreads);
    if (a.cols % (16 / sizeof(T)) == 0) k_norm_forward<T, kTpr, kNv, true><<<grid, block, 0, s>>>(a);
    else k_norm_forward<T, kTpr, kNv, false><<<grid, block, 0, s>>>(a);
}

template <typename T> void forward_of(const NormForward& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int64_t vecs = ceil_div(a.cols, V);
    if (a.cols < V) k_norm_forward_short<T><<<dim3((unsigned)std::min(ceil_div(a.rows, kShortBlock), kForwardThreads / kShortBlock)), dim3(kShortBlock), 0, s>>>(a);
    else if (vecs > 4096) k_norm_forward_long<T><<<dim3((unsigned)std::min(a.rows, kMaxNormBlocks)), dim3(1024), 0, s>>>(a);
    else if (vecs <= 16) forward_as<T, 16, 1>(a, s);
    else if (vecs <= 64) forward_as<T, 64, 1>(a, s);
    else if (vecs <= 128) forward_as<T, 64, 2>(a, s);
    else if (vecs <= 256) forward_as<T, 256, 1>(a, s);
    else if (vecs <= 512) forward_as<T, 256, 2>(a, s);
    else if (vecs <= 1024) forward_as<T, 512, 2>(a, s);
    else forward_as<T, 1024, 4>(a, s);
}

// Threads and vectors of a row in the backward pass; 0: too long for registers; 1 thread: shorter than a vector.
struct BackShape { int tpr, nv; };
BackShape back_shape(int64_t cols, int64_t v) {
    const int64_t vecs = ceil_div(cols, v);
    if (cols < v) return {1, 0};
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
    const int64_t groups = f.tpr == 1 ? ceil_div(rows, kShortBlock) : f.tpr ? ceil_div(rows, kBackBlock / f.tpr) : rows;
    return std::max<int64_t>(1, std::min(groups, kBackBlocks));
}

template <typename T> hipError_t backward_of(const NormBackward& a, hipStream_t s) {
    const BackShape f = back_shape(a.cols, 16 / (int64_t)sizeof(T));
    const int64_t blocks = back_blocks(a.rows, a.cols, sizeof(T));
    if (a.rows > 0) {
        switch (f.tpr * 8 + f.nv) {
            case 1 * 8: k_norm_backward_short<T><<<dim3((unsigned)blocks), dim3(kShortBlock), 0, s>>>(a); break;
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
        k_norm_weight_grad<<<dim3((unsigned)ceil_div(a.cols, kSumColumns), 2), dim3(1024), 0, s>>>(a.partial, a.rows > 0 ? blocks : 0, a.cols, a.dweight, a.dbias, a.weight_type);
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
