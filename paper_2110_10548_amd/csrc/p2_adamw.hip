// AdamW over many tensors at once, the sum of squares that clips it, and the values of 8-bit states.
//
// A launch takes up to kTensors tensors by value and one block for each kChunk values of them, so that nothing has to be copied to the device before a
// step, and a captured step keeps its tensors.
#include <algorithm>
#include <cstring>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kBlock = 256;
constexpr int kEach = 8;                       // values of a thread; 32 threads have a block of 8-bit states
constexpr int kChunk = kBlock * kEach;
constexpr int kTensors = 48;                   // kernel arguments are 4 KiB at most
constexpr int kSumTensors = 160;
constexpr int kSumBlocks = 1024;
static_assert(P2_STATE_BLOCK == 32 * kEach, "half a wavefront has a block of states");

template <int kMost, typename Entry> struct Table {
    Entry tensor[kMost];
    int32_t begin[kMost + 1];                  // the first chunk of each; the last one: all of them
    int32_t n;
};
template <typename Tab> __device__ __forceinline__ int tensor_of(const Tab& t, int chunk) {
    int low = 0, high = t.n - 1;
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (t.begin[mid] <= chunk) low = mid;
        else high = mid - 1;
    }
    return low;
}

struct SumEntry { const void* p; int64_t count; };
typedef Table<kSumTensors, SumEntry> SumTable;

__device__ __forceinline__ double block_sum(double v, double* buf) {       // thread 0 gets it
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v += buf[w];
    return v;
}

// Squares are added up in 64 bits: gradients of any size, and no overflow before the root.
template <typename T> __global__ __launch_bounds__(kBlock) void k_square_sum(SumTable table, double* parts) {
    __shared__ double buf[kBlock / 64];
    double s = 0.0;
    const int chunks = table.begin[table.n];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int i = tensor_of(table, c);
        const int64_t at = (int64_t)(c - table.begin[i]) * kChunk + threadIdx.x * kEach;
        float v[kEach];
        load_part<T, kEach>(static_cast<const T*>(table.tensor[i].p) + at, table.tensor[i].count - at, v, 0.0f);
#pragma unroll
        for (int j = 0; j < kEach; ++j) s += (double)v[j] * (double)v[j];
    }
    s = block_sum(s, buf);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}
__global__ __launch_bounds__(1024) void k_square_join(const double* parts, int64_t n, double* out) {
    __shared__ double buf[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += parts[i];
    s = block_sum(s, buf);
    if (threadIdx.x == 0) out[0] = s;
}

__global__ void k_adamw_numbers(Adamw a) {
    AdamwStep r = {};
    double factor = a.grad_factor;
    if (a.square_sum) {
        const double sum = a.square_sum[0];
        r.left_out = !(sum >= 0.0 && sum < __builtin_huge_val());
        factor *= fmin(1.0, a.max_norm / (a.grad_factor * sqrt(sum)));
    }
    if (!r.left_out) {
        const int64_t t = a.step[0] + 1;
        a.step[0] = t;
        const double lr = a.lr * (a.rate ? (double)a.rate[0] : 1.0);
        r.factor = (float)factor;
        r.rate = (float)(lr / (1.0 - pow(a.beta1, (double)t)));
        r.root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)t)));
        r.shrink = (float)(1.0 - lr * a.weight_decay);
    }
    a.numbers[0] = r;
}

// 8-bit states.  Each operation is rounded by itself (no multiply-adds): next to the border between two stored numbers everybody who
// follows the formula in 32 bits has the same one.
constexpr float kLeast = 0x1p-100f;

__device__ __forceinline__ float mean_of(int q, float scale) {
#pragma clang fp contract(off)
    return (float)(q * abs(q)) * (scale * (1.0f / 16129.0f));
}
__device__ __forceinline__ float square_of(int q, float scale) {
#pragma clang fp contract(off)
    const float r = (float)(q * q);
    return (r * (scale * (1.0f / 65025.0f))) * (r * (1.0f / 65025.0f));
}
// The largest absolute value of half a wavefront's, which is a block: NaN and infinities above everything.
__device__ __forceinline__ float block_scale(const float (&v)[kEach]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = group_reduce<32>(m, [](uint32_t x, uint32_t y) { return max(x, y); });
    const float s = __uint_as_float(m);
    return s < kLeast ? 0.0f : m >= 0x7f800000u ? __builtin_nanf("") : s;
}
__device__ __forceinline__ int mean_stored(float v, float inverse) {
#pragma clang fp contract(off)
    const float q = rintf(127.0f * sqrtf(fabsf(v) * inverse));
    return v < 0.0f ? -(int)q : (int)q;
}
__device__ __forceinline__ int square_stored(float v, float inverse) {
#pragma clang fp contract(off)
    const int q = (int)rintf(255.0f * sqrtf(sqrtf(v * inverse)));
    return v > 0.0f && inverse > 0.0f ? max(q, 1) : q;
}
__device__ __forceinline__ float inverse_of(float scale) { return scale > 0.0f ? 1.0f / scale : 0.0f; }      // (0, too, where it is NaN)

typedef Table<kTensors, p2_adamw_tensor> AdamwTable;
struct AdamwConstants { float beta1, beta2, rest1, rest2, eps; int32_t copy_type; };

typedef uint8_t bytes8 __attribute__((ext_vector_type(8), aligned(1)));

__device__ __forceinline__ void load_bytes(const uint8_t* p, int64_t n, uint8_t (&v)[kEach]) {
    if (n >= kEach) {
        const bytes8 r = *reinterpret_cast<const bytes8*>(p);
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = r[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = i < n ? p[i] : 0;
}
__device__ __forceinline__ void store_bytes(uint8_t* p, int64_t n, const uint8_t (&v)[kEach]) {
    if (n >= kEach) {
        bytes8 r;
#pragma unroll
        for (int i = 0; i < kEach; ++i) r[i] = v[i];
        *reinterpret_cast<bytes8*>(p) = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) if (i < n) p[i] = v[i];
}

template <typename P, typename G, int kBits> __global__ __launch_bounds__(kBlock) void k_adamw(AdamwTable table, AdamwConstants c, const AdamwStep* numbers) {
#pragma clang fp contract(off)
    const AdamwStep step = numbers[0];
    if (step.left_out) return;
    const int i = tensor_of(table, blockIdx.x);
    const p2_adamw_tensor& t = table.tensor[i];
    const int64_t at = (int64_t)((int)blockIdx.x - table.begin[i]) * kChunk + threadIdx.x * kEach, left = t.count - at;
    float p[kEach], g[kEach], m[kEach], v[kEach];
    load_part<P, kEach>(static_cast<const P*>(t.param) + at, left, p, 0.0f);
    load_part<G, kEach>(static_cast<const G*>(t.grad) + at, left, g, 0.0f);
    const int64_t block = at / P2_STATE_BLOCK;
    if constexpr (kBits == 8) {
        uint8_t q[kEach], r[kEach];
        load_bytes(static_cast<const uint8_t*>(t.mean) + at, left, q);
        load_bytes(static_cast<const uint8_t*>(t.square) + at, left, r);
        const float ms = left > 0 ? t.mean_scale[block] : 0.0f, ss = left > 0 ? t.square_scale[block] : 0.0f;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            m[j] = mean_of((int8_t)q[j], ms);
            v[j] = square_of(r[j], ss);
        }
    } else {
        load_part<float, kEach>(static_cast<const float*>(t.mean) + at, left, m, 0.0f);
        load_part<float, kEach>(static_cast<const float*>(t.square) + at, left, v, 0.0f);
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const float d = g[j] * step.factor;
        m[j] = c.beta1 * m[j] + c.rest1 * d;
        v[j] = c.beta2 * v[j] + c.rest2 * (d * d);
        p[j] = p[j] * step.shrink - step.rate * (m[j] / (sqrtf(v[j]) * step.root + c.eps));
    }
    store_part<P, kEach>(static_cast<P*>(t.param) + at, left, p);
    if (t.copy) {
        if (c.copy_type == P2_F32) store_part<float, kEach>(static_cast<float*>(t.copy) + at, left, p);
        else if (c.copy_type == P2_BF16) store_part<bf16_t, kEach>(static_cast<bf16_t*>(t.copy) + at, left, p);
        else store_part<half_t, kEach>(static_cast<half_t*>(t.copy) + at, left, p);
    }
    if constexpr (kBits == 8) {
        // (values past the tensor's end are zeros still)
        const float ms = block_scale(m), ss = block_scale(v), mi = inverse_of(ms), si = inverse_of(ss);
        uint8_t q[kEach], r[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            q[j] = mi > 0.0f ? (uint8_t)mean_stored(m[j], mi) : 0;
            r[j] = si > 0.0f ? (uint8_t)square_stored(v[j], si) : 0;
        }
        store_bytes(static_cast<uint8_t*>(t.mean) + at, left, q);
        store_bytes(static_cast<uint8_t*>(t.square) + at, left, r);
        if (threadIdx.x % 32 == 0 && left > 0) { t.mean_scale[block] = ms; t.square_scale[block] = ss; }
    } else {
        store_part<float, kEach>(static_cast<float*>(t.mean) + at, left, m);
        store_part<float, kEach>(static_cast<float*>(t.square) + at, left, v);
    }
}

__global__ __launch_bounds__(kBlock) void k_adamw_values(AdamwTable table) {
    const int i = tensor_of(table, blockIdx.x);
    const p2_adamw_tensor& t = table.tensor[i];            // (param and copy: where the values go)
    const int64_t at = (int64_t)((int)blockIdx.x - table.begin[i]) * kChunk + threadIdx.x * kEach, left = t.count - at;
    if (left <= 0) return;
    const int64_t block = at / P2_STATE_BLOCK;
    uint8_t q[kEach];
    float x[kEach];
    if (t.param) {
        load_bytes(static_cast<const uint8_t*>(t.mean) + at, left, q);
        const float s = t.mean_scale[block];
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] = mean_of((int8_t)q[j], s);
        store_part<float, kEach>(static_cast<float*>(t.param) + at, left, x);
    }
    if (t.copy) {
        load_bytes(static_cast<const uint8_t*>(t.square) + at, left, q);
        const float s = t.square_scale[block];
#pragma unroll
        for (int j = 0; j < kEach; ++j) x[j] = square_of(q[j], s);
        store_part<float, kEach>(static_cast<float*>(t.copy) + at, left, x);
    }
}

// Fills tables with the tensors that have values, and launches each.  (2^40 values are the most that a call takes: their chunks can be counted.)
template <typename Tab, typename Get, typename Launch> hipError_t in_tables(int64_t n, int most, Get&& get, Launch&& launch) {
    Tab table;
    table.n = 0;
    table.begin[0] = 0;
    for (int64_t i = 0; i < n; ++i) {
        const int64_t chunks = get(i, table.tensor[table.n]);
        if (chunks > 0) {
            table.begin[table.n + 1] = table.begin[table.n] + (int32_t)chunks;
            ++table.n;
        }
        if (table.n == most || (i + 1 == n && table.n > 0)) {
            launch(table);
            table.n = 0;
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <typename P, typename G> void step_launch(const AdamwTable& table, const AdamwConstants& c, int32_t bits, const AdamwStep* numbers, hipStream_t s) {
    const dim3 grid((unsigned)table.begin[table.n]);
    if (bits == 8) k_adamw<P, G, 8><<<grid, dim3(kBlock), 0, s>>>(table, c, numbers);
    else k_adamw<P, G, 32><<<grid, dim3(kBlock), 0, s>>>(table, c, numbers);
}
template <typename P> void step_launch(const AdamwTable& table, const AdamwConstants& c, int32_t grad_type, int32_t bits, const AdamwStep* numbers, hipStream_t s) {
    if (grad_type == P2_F32) step_launch<P, float>(table, c, bits, numbers, s);
    else if (grad_type == P2_BF16) step_launch<P, bf16_t>(table, c, bits, numbers, s);
    else step_launch<P, half_t>(table, c, bits, numbers, s);
}

}  // namespace

int64_t square_sum_parts(int64_t n) { return std::max<int64_t>(1, ceil_div(n, kSumTensors)) * kSumBlocks; }

hipError_t launch_square_sum(const void* const* tensors, const int64_t* counts, int64_t n, int32_t type, double* out, double* parts, hipStream_t s) {
    int64_t lines = 0;
    const hipError_t e = in_tables<SumTable>(
        n, kSumTensors,
        [&](int64_t i, SumEntry& t) {
            t = {tensors[i], counts[i]};
            return ceil_div(counts[i], kChunk);
        },
        [&](const SumTable& table) {
            const int blocks = std::min(table.begin[table.n], kSumBlocks);
            if (type == P2_F32) k_square_sum<float><<<dim3(blocks), dim3(kBlock), 0, s>>>(table, parts + lines);
            else if (type == P2_BF16) k_square_sum<bf16_t><<<dim3(blocks), dim3(kBlock), 0, s>>>(table, parts + lines);
            else k_square_sum<half_t><<<dim3(blocks), dim3(kBlock), 0, s>>>(table, parts + lines);
            lines += blocks;
        });
    if (e != hipSuccess) return e;
    k_square_join<<<dim3(1), dim3(1024), 0, s>>>(parts, lines, out);
    return hipGetLastError();
}

hipError_t launch_adamw(const Adamw& a, hipStream_t s) {
    k_adamw_numbers<<<dim3(1), dim3(1), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const AdamwConstants c = {(float)a.beta1, (float)a.beta2, (float)(1.0 - a.beta1), (float)(1.0 - a.beta2), (float)a.eps, a.copy_type};
    return in_tables<AdamwTable>(
        a.n, kTensors,
        [&](int64_t i, p2_adamw_tensor& t) {
            t = a.tensors[i];
            return ceil_div(t.count, kChunk);
        },
        [&](const AdamwTable& table) {
            if (a.type == P2_F32) step_launch<float>(table, c, a.grad_type, a.state_bits, a.numbers, s);
            else if (a.type == P2_BF16) step_launch<bf16_t>(table, c, a.grad_type, a.state_bits, a.numbers, s);
            else step_launch<half_t>(table, c, a.grad_type, a.state_bits, a.numbers, s);
        });
}

hipError_t launch_adamw_values(const p2_adamw_tensor* tensors, int64_t n, float* const* mean_out, float* const* square_out, hipStream_t s) {
    return in_tables<AdamwTable>(
        n, kTensors,
        [&](int64_t i, p2_adamw_tensor& t) {
            t = tensors[i];
            t.param = mean_out ? mean_out[i] : nullptr;
            t.copy = square_out ? square_out[i] : nullptr;
            return t.param || t.copy ? ceil_div(t.count, kChunk) : 0;
        },
        [&](const AdamwTable& table) { k_adamw_values<<<dim3((unsigned)table.begin[table.n]), dim3(kBlock), 0, s>>>(table); });
}

}  // namespace p2
