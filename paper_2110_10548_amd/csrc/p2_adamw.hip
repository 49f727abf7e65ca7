// AdamW over many tensors at once, the sum of squares that clips it, and the values of 8-bit states.
//
// A launch takes up to kTensors tensors by value and one block for each kChunk values of them, so that nothing has to be copied to the device before a
// step, and a captured step keeps its tensors.
#include <algorithm>
#include <cmath>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kBlock = 256;
constexpr int kEach = 8;                       // values of a thread; 32 threads have a block of 8-bit states
constexpr int kChunk = kBlock * kEach;
constexpr int kTensors = 48;                   // kernel arguments are 4 KiB at most
constexpr int kSumTensors = 160;
constexpr int kSumBlocks = 2048, kSumChunk = kBlock * 32, kSumAlone = 32;     // (kSumAlone chunks at most: one block of 1024 threads has them)
static_assert(P2_STATE_BLOCK == 32 * kEach, "half a wavefront has a block of states");

template <int kMost, typename Entry> struct Table {
    Entry tensor[kMost];
    int32_t begin[kMost + 1];                  // the first chunk of each; the last one: all of them
    int32_t n;
};
// The tensor of a chunk, the same for the whole wavefront: a look at all of them at once (a search would wait for six loads, one after the other).
template <int kMost> __device__ __forceinline__ int tensor_of(const int32_t* begin, int n, int chunk) {
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int base = 0; base < kMost; base += 64) {
        const int i = base + lane;
        before += __popcll(__ballot(i < n && begin[min(i, n)] <= chunk));
    }
    return __builtin_amdgcn_readfirstlane(before - 1);
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

// Squares are added up in 64 bits: gradients of any size, and no overflow before the root.  A block of kThreads takes chunks of kSumChunk values, four vectors a thread
// at a time.  Where one block has all of them it writes the sum itself.
template <typename T, int kThreads> __global__ __launch_bounds__(kThreads) void k_square_sum(SumTable table, double* parts) {
    constexpr int V = kSumChunk / kBlock / 4;
    __shared__ double buf[kThreads / 64];
    // (looked up in LDS: a load from memory would have to wait for the values asked for before it)
    __shared__ int32_t begins[kSumTensors + 1];
    for (int i = threadIdx.x; i <= table.n; i += kThreads) begins[i] = table.begin[i];
    __syncthreads();
    double s = 0.0;
    const int chunks = table.begin[table.n], each = kThreads / kBlock, x = threadIdx.x % kBlock;
    // A chunk is asked for while the one before it is added up.
    vec_t<T, V> next[4] = {};
    const auto ask = [&](int c) {
        const int i = tensor_of<kSumTensors>(begins, table.n, c);
        const int64_t at = (int64_t)(c - table.begin[i]) * kSumChunk, left = table.tensor[i].count - at;
        const T* p = static_cast<const T*>(table.tensor[i].p) + at;
        if (left >= kSumChunk) {
#pragma unroll
            for (int q = 0; q < 4; ++q) next[q] = *reinterpret_cast<const vec_t<T, V>*>(p + (q * kBlock + x) * V);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t e = (q * kBlock + x) * V;
                if (left - e >= V) {
                    next[q] = *reinterpret_cast<const vec_t<T, V>*>(p + e);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) next[q][j] = (T)0.0f;
                    for (int j = 0; e + j < left; ++j)
#pragma unroll
                        for (int w = 0; w < V; ++w)
                            if (w == j) next[q][w] = p[e + j];
                }
            }
        }
    };
    int c = blockIdx.x * each + threadIdx.x / kBlock;
    if (c < chunks) ask(c);
    while (c < chunks) {
        vec_t<T, V> v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = next[q];
        c += gridDim.x * each;
        if (c < chunks) ask(c);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < V; ++j) s = fma((double)(float)v[q][j], (double)(float)v[q][j], s);
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

// The largest absolute value of half a wavefront's, which is a block: NaN and infinities above everything.
__device__ __forceinline__ float block_scale(const float (&v)[kEach]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = group_reduce<32>(m, [](uint32_t x, uint32_t y) { return max(x, y); });
    const float s = __uint_as_float(m);
    return s < kLeast ? 0.0f : m >= 0x7f800000u ? __builtin_nanf("") : s;
}
// The number to store: the nearest one to 127 sqrt(|v| / scale) and 255 (v / scale)^(1/4), each root and product rounded to 32 bits.  The instruction for the root is
// off by a step at most where the function's is by half of one, so that the places differ by 127 * 2.5 * 2^-23 = 3.8e-5 and 255 * 3.25 * 2^-23 = 9.9e-5 at most; where that
// could matter, next to the middle of two numbers (one value in some 10000 and one in 4000), the wavefront works its roots out as they are defined (sqrtf: ten instructions).
constexpr float kNearMean = 0.5f - 4e-5f, kNearSquare = 0.5f - 1.1e-4f;

template <bool kExact> __device__ __forceinline__ float root_of(float v) { return kExact ? sqrtf(v) : __builtin_amdgcn_sqrtf(v); }
template <bool kSquare, bool kExact> __device__ __forceinline__ float place_of(float v, float inverse) {
#pragma clang fp contract(off)
    const float x = fabsf(v) * inverse;
    return kSquare ? 255.0f * root_of<kExact>(root_of<kExact>(x)) : 127.0f * root_of<kExact>(x);
}
// The numbers of eight values as bytes.
typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(1)));
template <bool kSquare> __device__ __forceinline__ words2 stored(const float (&v)[kEach], float inverse) {
    float q[kEach];
    bool near = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const float place = place_of<kSquare, false>(v[i], inverse);
        q[i] = __builtin_rintf(place);
        near |= fabsf(place - q[i]) > (kSquare ? kNearSquare : kNearMean);
    }
    if (__any(near))
#pragma unroll
        for (int i = 0; i < kEach; ++i) q[i] = __builtin_rintf(place_of<kSquare, true>(v[i], inverse));
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (kSquare) q[i] = v[i] > 0.0f ? fmaxf(q[i], 1.0f) : q[i];
        else q[i] = copysignf(q[i], v[i]) + 128.0f;        // (bytes without a sign are made in one instruction)
#if defined(__HIP_DEVICE_COMPILE__)
        w[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(q[i], i % 4, w[i / 4]);
#endif
    }
    const uint32_t sign = kSquare ? 0u : 0x80808080u;
    return inverse > 0.0f ? words2{w[0] ^ sign, w[1] ^ sign} : words2{0, 0};
}
__device__ __forceinline__ float inverse_of(float scale) { return scale > 0.0f ? 1.0f / scale : 0.0f; }      // (0, too, where it is NaN)

typedef Table<kTensors, p2_adamw_tensor> AdamwTable;
struct AdamwConstants { float beta1, beta2, rest1, rest2, eps; int32_t copy_type, by_instruction; };

// Eight stored numbers: bytes, as two words.  Means are stored as they are, of squares without a sign.
__device__ __forceinline__ words2 load_bytes(const void* p, int64_t n) {
    if (n >= kEach) return *static_cast<const words2*>(p);
    words2 r = {0, 0};
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (i < n) r[i / 4] |= (uint32_t)static_cast<const uint8_t*>(p)[i] << i % 4 * 8;
    return r;
}
__device__ __forceinline__ void store_bytes(void* p, int64_t n, words2 v) {
    if (n >= kEach) { *static_cast<words2*>(p) = v; return; }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (i < n) static_cast<uint8_t*>(p)[i] = (uint8_t)(v[i / 4] >> i % 4 * 8);
}
__device__ __forceinline__ void means_of(words2 q, float scale, float (&v)[kEach]) {
#pragma clang fp contract(off)
    const float unit = scale * (1.0f / 16129.0f);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const float f = (float)((q[i / 4] ^ 0x80808080u) >> i % 4 * 8 & 0xffu) - 128.0f;       // (an unsigned byte is converted in one instruction)
        v[i] = f * fabsf(f) * unit;
    }
}
__device__ __forceinline__ void squares_of(words2 q, float scale, float (&v)[kEach]) {
#pragma clang fp contract(off)
    const float unit = scale * (1.0f / 65025.0f);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const float f = (float)(q[i / 4] >> i % 4 * 8 & 0xffu), r = f * f;
        v[i] = (r * unit) * (r * (1.0f / 65025.0f));
    }
}

template <typename P, typename G, int kBits> __device__ __forceinline__ void adamw_chunk(const AdamwTable& table, const AdamwConstants& c, const AdamwStep& step, int chunk) {
#pragma clang fp contract(off)
    const int i = tensor_of<kTensors>(table.begin, table.n, chunk);
    const p2_adamw_tensor& t = table.tensor[i];
    const int64_t at = (int64_t)(chunk - table.begin[i]) * kChunk + threadIdx.x * kEach, left = t.count - at;
    float p[kEach], g[kEach], m[kEach], v[kEach];
    load_part<P, kEach>(static_cast<const P*>(t.param) + at, left, p, 0.0f);
    load_part<G, kEach>(static_cast<const G*>(t.grad) + at, left, g, 0.0f);
    const int64_t block = at / P2_STATE_BLOCK;
    if constexpr (kBits == 8) {
        const words2 q = load_bytes(static_cast<const uint8_t*>(t.mean) + at, left), r = load_bytes(static_cast<const uint8_t*>(t.square) + at, left);
        const float ms = left > 0 ? t.mean_scale[block] : 0.0f, ss = left > 0 ? t.square_scale[block] : 0.0f;
        means_of(q, ms, m);
        squares_of(r, ss, v);
    } else {
        load_part<float, kEach>(static_cast<const float*>(t.mean) + at, left, m, 0.0f);
        load_part<float, kEach>(static_cast<const float*>(t.square) + at, left, v, 0.0f);
    }
    float update[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const float d = g[j] * step.factor;
        m[j] = c.beta1 * m[j] + c.rest1 * d;
        v[j] = c.beta2 * v[j] + c.rest2 * (d * d);
    }
    // The instructions for the root and 1 / x are off by a step each, 2^-22 of the update.
    if (c.by_instruction) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) update[j] = m[j] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[j]) * step.root + c.eps);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j) update[j] = m[j] / (sqrtf(v[j]) * step.root + c.eps);
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) p[j] = p[j] * step.shrink - step.rate * update[j];
    store_part<P, kEach>(static_cast<P*>(t.param) + at, left, p);
    if (t.copy) {
        if (c.copy_type == P2_F32) store_part<float, kEach>(static_cast<float*>(t.copy) + at, left, p);
        else if (c.copy_type == P2_BF16) store_part<bf16_t, kEach>(static_cast<bf16_t*>(t.copy) + at, left, p);
        else store_part<half_t, kEach>(static_cast<half_t*>(t.copy) + at, left, p);
    }
    if constexpr (kBits == 8) {
        // (values past the tensor's end are zeros still)
        const float ms = block_scale(m), ss = block_scale(v), mi = inverse_of(ms), si = inverse_of(ss);
        const words2 q = stored<false>(m, mi), r = stored<true>(v, si);
        store_bytes(static_cast<uint8_t*>(t.mean) + at, left, q);
        store_bytes(static_cast<uint8_t*>(t.square) + at, left, r);
        if (threadIdx.x % 32 == 0 && left > 0) { t.mean_scale[block] = ms; t.square_scale[block] = ss; }
    } else {
        store_part<float, kEach>(static_cast<float*>(t.mean) + at, left, m);
        store_part<float, kEach>(static_cast<float*>(t.square) + at, left, v);
    }
}

template <typename P, typename G, int kBits> __global__ __launch_bounds__(kBlock) void k_adamw(AdamwTable table, AdamwConstants c, const AdamwStep* numbers) {
    const AdamwStep step = numbers[0];
    if (step.left_out) return;
    for (int chunk = blockIdx.x; chunk < table.begin[table.n]; chunk += gridDim.x) adamw_chunk<P, G, kBits>(table, c, step, chunk);
}

__device__ __forceinline__ void values_of_chunk(const AdamwTable& table, int chunk) {
    const int i = tensor_of<kTensors>(table.begin, table.n, chunk);
    const p2_adamw_tensor& t = table.tensor[i];            // (param and copy: where the values go)
    const int64_t at = (int64_t)(chunk - table.begin[i]) * kChunk + threadIdx.x * kEach, left = t.count - at;
    if (left <= 0) return;
    const int64_t block = at / P2_STATE_BLOCK;
    float x[kEach];
    if (t.param) {
        means_of(load_bytes(static_cast<const uint8_t*>(t.mean) + at, left), t.mean_scale[block], x);
        store_part<float, kEach>(static_cast<float*>(t.param) + at, left, x);
    }
    if (t.copy) {
        squares_of(load_bytes(static_cast<const uint8_t*>(t.square) + at, left), t.square_scale[block], x);
        store_part<float, kEach>(static_cast<float*>(t.copy) + at, left, x);
    }
}

__global__ __launch_bounds__(kBlock) void k_adamw_values(AdamwTable table) {
    for (int chunk = blockIdx.x; chunk < table.begin[table.n]; chunk += gridDim.x) values_of_chunk(table, chunk);
}

// (a launch has less than 2^32 threads)
dim3 chunks_of(const AdamwTable& table) { return dim3((unsigned)std::min(table.begin[table.n], 1 << 23)); }

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
    const dim3 grid = chunks_of(table);
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

template <typename T> static hipError_t square_sum(const void* const* tensors, const int64_t* counts, int64_t n, double* out, double* parts, hipStream_t s) {
    int64_t lines = 0, chunks = 0;
    for (int64_t i = 0; i < n; ++i) chunks += ceil_div(counts[i], kSumChunk);
    const bool alone = chunks > 0 && chunks <= kSumAlone && n <= kSumTensors;
    const hipError_t e = in_tables<SumTable>(
        n, kSumTensors,
        [&](int64_t i, SumEntry& t) {
            t = {tensors[i], counts[i]};
            return ceil_div(counts[i], kSumChunk);
        },
        [&](const SumTable& table) {
            const int blocks = alone ? 1 : std::min(table.begin[table.n], kSumBlocks);
            if (alone) k_square_sum<T, 1024><<<dim3(1), dim3(1024), 0, s>>>(table, out);
            else k_square_sum<T, kBlock><<<dim3(blocks), dim3(kBlock), 0, s>>>(table, parts + lines);
            lines += blocks;
        });
    if (e != hipSuccess || alone) return e;
    k_square_join<<<dim3(1), dim3(1024), 0, s>>>(parts, lines, out);
    return hipGetLastError();
}

hipError_t launch_square_sum(const void* const* tensors, const int64_t* counts, int64_t n, int32_t type, double* out, double* parts, hipStream_t s) {
    return type == P2_F32 ? square_sum<float>(tensors, counts, n, out, parts, s) : type == P2_BF16 ? square_sum<bf16_t>(tensors, counts, n, out, parts, s) : square_sum<half_t>(tensors, counts, n, out, parts, s);
}

hipError_t launch_adamw(const Adamw& a, hipStream_t s) {
    k_adamw_numbers<<<dim3(1), dim3(1), 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // (The root's instruction takes squares below 2^-126 for 0.  Their roots are 2^-63 at most, and root is at most 1 / sqrt(1 - beta2): 2^-24 of such an eps.)
    const bool by_instruction = a.eps * std::sqrt(1.0 - a.beta2) >= 0x1p-39;
    const AdamwConstants c = {(float)a.beta1, (float)a.beta2, (float)(1.0 - a.beta1), (float)(1.0 - a.beta2), (float)a.eps, a.copy_type, by_instruction};
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
        [&](const AdamwTable& table) { k_adamw_values<<<chunks_of(table), dim3(kBlock), 0, s>>>(table); });
}

}  // namespace p2
