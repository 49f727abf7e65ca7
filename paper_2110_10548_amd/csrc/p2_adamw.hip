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
constexpr int kSumBlocks = 2048, kSumChunk = kBlock * 32;
constexpr int kSumPiece = 512, kSumAlone = 512;    // one block of 16 wavefronts has up to kSumAlone pieces; a lane looks up one of its wavefront's
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

// Squares are added up in 64 bits: gradients of any size, and no overflow before the root.  A block takes chunks of kSumChunk values, four vectors a thread at a time.
// Bound by memory: 0.1 billion bf16 values 46 us, 4.4 TB/s, and 4.6 for the launch that joins the blocks' sums (39 for both behind themselves, part of the values from the last cache).
template <typename T> __global__ __launch_bounds__(kBlock) void k_square_sum(SumTable table, double* parts) {
    constexpr int V = kSumChunk / kBlock / 4;
    __shared__ double buf[kBlock / 64];
    // (looked up in LDS: a load from memory would have to wait for the values asked for before it)
    __shared__ int32_t begins[kSumTensors + 1];
    for (int i = threadIdx.x; i <= table.n; i += kBlock) begins[i] = table.begin[i];
    __syncthreads();
    double s = 0.0;
    const int chunks = table.begin[table.n], x = threadIdx.x;
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
    int c = blockIdx.x;
    if (c < chunks) ask(c);
    while (c < chunks) {
        vec_t<T, V> v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = next[q];
        c += gridDim.x;
        if (c < chunks) ask(c);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < V; ++j) s = fma((double)(float)v[q][j], (double)(float)v[q][j], s);
    }
    s = block_sum(s, buf);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The same for few values, by one block, which writes the sum itself: latency is all it takes, so a wavefront's pieces of kSumPiece values are looked up by its lanes at
// once, and eight of them are under way together (0.1 million fp32 values in 20 tensors: 8.1 us; by chunks, one ahead, 11.7).
template <typename T> __global__ __launch_bounds__(1024) void k_square_few(SumTable table, double* out) {
    constexpr int V = kSumPiece / 64, kAhead = 8;
    __shared__ double buf[16];
    __shared__ int32_t begins[kSumTensors + 1];
    __shared__ SumEntry tensors[kSumTensors];
    for (int i = threadIdx.x; i <= table.n; i += 1024) {
        begins[i] = table.begin[i];
        if (i < table.n) tensors[i] = table.tensor[i];
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pieces = begins[table.n];
    // lane l: where the wavefront's l-th piece lies, and how much of it there is
    const int piece = wave + 16 * lane;
    int low = 0, high = table.n;                               // begins[low] <= piece
    while (high - low > 1) {
        const int middle = (low + high) / 2;
        if (begins[middle] <= piece) low = middle;
        else high = middle;
    }
    const int64_t at = (int64_t)(piece - begins[low]) * kSumPiece;
    const uint64_t where = reinterpret_cast<uint64_t>(static_cast<const T*>(tensors[low].p) + at);
    const int size = piece < pieces ? (int)min(tensors[low].count - at, (int64_t)kSumPiece) : 0;
    const int mine = pieces > wave ? (pieces - wave + 15) / 16 : 0;
    double s = 0.0;
    for (int first = 0; first < mine; first += kAhead) {
        vec_t<T, V> v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int from = min(first + u, 63);               // (a piece past the last has no values)
            const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(where >> 32), from) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)where, from);
            const int left = (first + u < 64 ? __builtin_amdgcn_readlane(size, from) : 0) - lane * V;
            const T* p = reinterpret_cast<const T*>(base) + lane * V;
#pragma unroll
            for (int j = 0; j < V; ++j) v[u][j] = (T)0.0f;
            if (left >= V) {
                v[u] = *reinterpret_cast<const vec_t<T, V>*>(p);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j < left) v[u][j] = p[j];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int j = 0; j < V; ++j) s = fma((double)(float)v[u][j], (double)(float)v[u][j], s);
    }
    s = block_sum(s, buf);
    if (threadIdx.x == 0) out[0] = s;
}
__global__ __launch_bounds__(1024) void k_square_join(const double* parts, int64_t n, double* out) {
    __shared__ double buf[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += parts[i];
    s = block_sum(s, buf);
    if (threadIdx.x == 0) out[0] = s;
}

// b^t for b in [0, 1): what the squarings round off, t 2^-53 of it, is less than 2^-53 / (1 - b) of anything.
__device__ __forceinline__ double power(double b, int64_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return r;
}
// The numbers of step t, by a whole wavefront: latency is all they take, so the betas' powers are two lanes'.  (A t outside 1 to 2^40 - 1, as of a negative step, is no step's.)
constexpr int kStepBits = 40;
__device__ __forceinline__ AdamwStep numbers_of(const AdamwCall& a, int64_t t) {
    AdamwStep r = {};
    r.left_out = t < 1 || t >> kStepBits != 0;
    const double left = 1.0 - power((threadIdx.x & 1) == 0 ? a.beta1 : a.beta2, t), left1 = __shfl(left, 0, 64), left2 = __shfl(left, 1, 64);
    double factor = a.grad_factor;
    if (a.square_sum) {
        const double sum = a.square_sum[0];
        r.left_out |= !(sum >= 0.0 && sum < __builtin_huge_val());
        factor *= fmin(1.0, a.max_norm / (a.grad_factor * sqrt(sum)));
    }
    const double lr = a.lr * (a.rate ? (double)a.rate[0] : 1.0);
    r.factor = (float)factor;
    r.rate = (float)(lr / left1);
    r.root = (float)(1.0 / sqrt(left2));
    r.shrink = (float)(1.0 - lr * a.weight_decay);
    return r;
}
__global__ __launch_bounds__(64) void k_adamw_numbers(AdamwCall a, AdamwStep* numbers) {
    const int64_t t = a.step[0] < 0 ? 0 : a.step[0] + 1;
    const AdamwStep r = numbers_of(a, t);
    if (threadIdx.x != 0) return;
    numbers[0] = r;
    if (!r.left_out) a.step[0] = t;
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

// Values for which the caches have no use: the values of 0.1 billion 8-bit states take 204 us by themselves instead of 238, 226 behind a step.
typedef float float4_a __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void store_past(float* p, int64_t n, const float (&v)[kEach]) {
    if (n < kEach) { store_part<float, kEach>(p, n, v); return; }
#pragma unroll
    for (int q = 0; q < kEach / 4; ++q) __builtin_nontemporal_store(float4_a{v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]}, reinterpret_cast<float4_a*>(p + q * 4));
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

// Bound by memory, each value read and written once: 0.2 billion fp32 weights with bf16 gradients and copies 1044 us, 5.4 TB/s; 0.1 billion bf16 weights with 8-bit states 183 us, 5.6 TB/s.
// A block has 2048 values, eight a thread, so that half a wavefront has the 256 values of a scale.
template <typename P, typename G, int kBits> __global__ __launch_bounds__(kBlock) void k_adamw(AdamwTable table, AdamwConstants c, const AdamwStep* numbers) {
    const AdamwStep step = numbers[0];
    if (step.left_out) return;
    for (int chunk = blockIdx.x; chunk < table.begin[table.n]; chunk += gridDim.x) adamw_chunk<P, G, kBits>(table, c, step, chunk);
}

// A step of one launch with a block a chunk works out the numbers itself, in every wavefront, which saves the launch before it (0.1 million values in 20 tensors with
// their sum of squares: 20.9 -> 17.3 us, both calls, of which 16 are the host's; above kAlone chunks it is not noticed).  step[0] may become t once every block has read it: blocks that are done count themselves
// in its upper bits, which nothing else uses, and the last one writes t.
constexpr int kAlone = 1024;
template <typename P, typename G, int kBits> __global__ __launch_bounds__(kBlock) void k_adamw_alone(AdamwTable table, AdamwConstants c, AdamwCall a) {
    const int64_t before = __hip_atomic_load(a.step, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), t = before < 0 ? 0 : (before & (((int64_t)1 << kStepBits) - 1)) + 1;
    const AdamwStep step = numbers_of(a, t);
    if (step.left_out) return;
    adamw_chunk<P, G, kBits>(table, c, step, blockIdx.x);
    __syncthreads();                                           // (all wavefronts have read it)
    if (threadIdx.x != 0) return;
    unsigned long long* const count = reinterpret_cast<unsigned long long*>(a.step);
    if (atomicAdd(count, 1ull << kStepBits) >> kStepBits == gridDim.x - 1) atomicExch(count, (unsigned long long)t);
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
        store_past(static_cast<float*>(t.param) + at, left, x);
    }
    if (t.copy) {
        squares_of(load_bytes(static_cast<const uint8_t*>(t.square) + at, left), t.square_scale[block], x);
        store_past(static_cast<float*>(t.copy) + at, left, x);
    }
}

// Bound by what is written: 0.1 billion values of each 226 us behind a step, 4.5 TB/s with what is read (204 by itself, 4.9).
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

template <typename P, typename G> void step_in(const AdamwTable& table, const AdamwConstants& c, const Adamw& a, bool alone, hipStream_t s) {
    const dim3 grid = chunks_of(table), block(kBlock);
    if (alone && a.state_bits == 8) k_adamw_alone<P, G, 8><<<grid, block, 0, s>>>(table, c, a.call);
    else if (alone) k_adamw_alone<P, G, 32><<<grid, block, 0, s>>>(table, c, a.call);
    else if (a.state_bits == 8) k_adamw<P, G, 8><<<grid, block, 0, s>>>(table, c, a.numbers);
    else k_adamw<P, G, 32><<<grid, block, 0, s>>>(table, c, a.numbers);
}
template <typename P> void step_launch(const AdamwTable& table, const AdamwConstants& c, const Adamw& a, bool alone, hipStream_t s) {
    if (a.grad_type == P2_F32) step_in<P, float>(table, c, a, alone, s);
    else if (a.grad_type == P2_BF16) step_in<P, bf16_t>(table, c, a, alone, s);
    else step_in<P, half_t>(table, c, a, alone, s);
}

}  // namespace

int64_t square_sum_parts(int64_t n) { return std::max<int64_t>(1, ceil_div(n, kSumTensors)) * kSumBlocks; }

template <typename T> static hipError_t square_sum(const void* const* tensors, const int64_t* counts, int64_t n, double* out, double* parts, hipStream_t s) {
    int64_t lines = 0, pieces = 0;
    for (int64_t i = 0; i < n; ++i) pieces += ceil_div(counts[i], kSumPiece);
    const bool alone = pieces > 0 && pieces <= kSumAlone && n <= kSumTensors;
    const hipError_t e = in_tables<SumTable>(
        n, kSumTensors,
        [&](int64_t i, SumEntry& t) {
            t = {tensors[i], counts[i]};
            return ceil_div(counts[i], alone ? kSumPiece : kSumChunk);
        },
        [&](const SumTable& table) {
            if (alone) { k_square_few<T><<<dim3(1), dim3(1024), 0, s>>>(table, out); return; }
            const int blocks = std::min(table.begin[table.n], kSumBlocks);
            k_square_sum<T><<<dim3(blocks), dim3(kBlock), 0, s>>>(table, parts + lines);
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
    int64_t used = 0, chunks = 0;
    for (int64_t i = 0; i < a.n; ++i) { used += a.tensors[i].count > 0; chunks += ceil_div(a.tensors[i].count, kChunk); }
    const bool alone = used > 0 && used <= kTensors && chunks <= kAlone;
    if (!alone) {
        k_adamw_numbers<<<dim3(1), dim3(64), 0, s>>>(a.call, a.numbers);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // (The root's instruction takes squares below 2^-126 for 0.  Their roots are 2^-63 at most, and root is at most 1 / sqrt(1 - beta2): 2^-24 of such an eps.)
    const bool by_instruction = a.eps * std::sqrt(1.0 - a.call.beta2) >= 0x1p-39;
    const AdamwConstants c = {(float)a.call.beta1, (float)a.call.beta2, (float)(1.0 - a.call.beta1), (float)(1.0 - a.call.beta2), (float)a.eps, a.copy_type, by_instruction};
    return in_tables<AdamwTable>(
        a.n, kTensors,
        [&](int64_t i, p2_adamw_tensor& t) {
            t = a.tensors[i];
            return ceil_div(t.count, kChunk);
        },
        [&](const AdamwTable& table) {
            if (a.type == P2_F32) step_launch<float>(table, c, a, alone, s);
            else if (a.type == P2_BF16) step_launch<bf16_t>(table, c, a, alone, s);
            else step_launch<half_t>(table, c, a, alone, s);
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
