// Routing to experts: scores (softmax or sigmoid), a choice by score + bias within the best groups, gates, counts; the gradient of the
// gates with respect to the logits; the biases' step.
//
// A token's logits stay in the registers of its lanes.  The lanes are dealt out to the groups: a group has kLanes / (groups rounded up to a
// power of two) of them, so that a group's value is a reduction over neighbouring lanes, and a lane holds values of one group alone.
#include <algorithm>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kBlock = 256;
constexpr int64_t kRouteBlocks = 1024;
constexpr float kLog2e = 1.44269504088896340736f;

// How a token's lanes and their values are dealt out.
struct Shape {
    int32_t lanes, items;              // of a token; of a lane
    int32_t group_lanes;               // lanes of a group
};
int32_t power_of_two(int64_t v) {
    int32_t p = 1;
    while (p < v) p *= 2;
    return p;
}
Shape shape_of(int32_t experts, int32_t k, int32_t groups) {
    const int32_t places = power_of_two(groups);
    const int64_t size = experts / groups;
    Shape s = {};
    for (s.items = experts <= 128 ? 8 : 16; s.items <= 32; s.items *= 2) {
        s.group_lanes = power_of_two(ceil_div(size, s.items));
        s.lanes = s.group_lanes * places;
        if (s.lanes <= 64) break;
    }
    while (s.lanes < k) { s.lanes *= 2; s.group_lanes *= 2; }      // lane i keeps the i-th choice
    return s;
}

// A 64-bit number's bits in its order; NaN above everything.  0: not on offer.
__device__ __forceinline__ uint64_t ordered(double v) {
    if (v != v) return ~0ull;
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
    return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(uint64_t k) {
    if (k == ~0ull) return __builtin_nan("");
    return __longlong_as_double((long long)(k & 0x8000000000000000ull ? k & 0x7fffffffffffffffull : ~k));
}

// A reduction over `lanes` neighbouring lanes, as many as the launch says.
template <typename V, typename F> __device__ __forceinline__ V over_lanes(V v, int lanes, F&& f) {
    for (int d = 1; d < lanes; d <<= 1) v = f(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ uint64_t larger(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t smaller(uint64_t a, uint64_t b) { return a < b ? a : b; }

// A lane's values of its group's part of a row.  Value i belongs to expert expert(i), or to none.
template <typename T, int kItems> struct Part {
    static constexpr int V = 16 / sizeof(T);
    int first, size, lane, lanes;              // the group's first expert and their number (0: no group); this lane's place in it
    __device__ __forceinline__ int at(int i) const { return ((i / V) * lanes + lane) * V; }
    __device__ __forceinline__ bool mine(int i) const { return at(i) + i % V < size; }
    __device__ __forceinline__ int expert(int i) const { return first + at(i) + i % V; }
    __device__ __forceinline__ void load(const T* row, float (&z)[kItems]) const {
#pragma unroll
        for (int q = 0; q < kItems / V; ++q) {
            float v[V];
            load_part<T, V>(row + first + at(q * V), size - at(q * V), v, -INFINITY);
#pragma unroll
            for (int j = 0; j < V; ++j) z[q * V + j] = v[j];
        }
    }
};

template <typename T, int kLanes, int kItems> __global__ __launch_bounds__(kBlock) void k_route_forward(RouteForward a, int32_t group_lanes) {
    constexpr int kTokens = kBlock / kLanes;
    __shared__ int32_t count[P2_MAX_EXPERTS + 1];
    const int lane = threadIdx.x % kLanes;
    for (int e = threadIdx.x; e <= a.experts; e += kBlock) count[e] = 0;
    __syncthreads();
    const int group = lane / group_lanes;
    Part<T, kItems> part;
    part.size = group < a.groups ? a.experts / a.groups : 0;
    part.first = group < a.groups ? group * part.size : 0;
    part.lane = lane % group_lanes;
    part.lanes = group_lanes;
    for (int64_t t0 = (int64_t)blockIdx.x * kTokens; t0 < a.tokens; t0 += (int64_t)gridDim.x * kTokens) {
        const int64_t t = t0 + threadIdx.x / kLanes;
        const bool there = t < a.tokens;
        const T* row = static_cast<const T*>(a.logits) + (there ? t : a.tokens - 1) * a.stride;
        float z[kItems];
        part.load(row, z);
        bool any = false;
#pragma unroll
        for (int i = 0; i < kItems; ++i) any |= part.mine(i) && z[i] != -INFINITY;
        any = group_reduce<kLanes>((uint32_t)any, [](uint32_t x, uint32_t y) { return x | y; }) != 0;
        const bool on = there && any && (!a.keep || a.keep[t]);
        // scores and what is chosen by
        double most = -INFINITY, inv = 1.0;
        if (a.score == P2_SOFTMAX) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < kItems; ++i) most = fmax(most, (double)z[i]);
            most = over_lanes(most, kLanes, [](double x, double y) { return fmax(x, y); });
#pragma unroll
            for (int i = 0; i < kItems; ++i) sum += exp((double)z[i] - most);
            sum = over_lanes(sum, kLanes, [](double x, double y) { return x + y; });
            inv = 1.0 / sum;
        }
        uint64_t key[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const double s = a.score == P2_SOFTMAX ? exp((double)z[i] - most) * inv : 1.0 / (1.0 + exp(-(double)z[i]));
            const bool mine = part.mine(i);
            const float b = mine && a.bias ? a.bias[part.expert(i)] : 0.0f;
            key[i] = on && mine && z[i] != -INFINITY && b != -INFINITY ? ordered(s + (double)b) : 0;
        }
        if (a.groups > 1) {
            uint64_t one = 0, two = 0;                         // the group's largest
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                two = larger(two, smaller(one, key[i]));
                one = larger(one, key[i]);
            }
            for (int d = 1; d < group_lanes; d <<= 1) {
                const uint64_t o = __shfl_xor(one, d, 64), w = __shfl_xor(two, d, 64);
                two = larger(larger(two, w), smaller(one, o));
                one = larger(one, o);
            }
            const uint64_t value = one == 0 || two == 0 || a.group_best == 1 ? one : ordered(value_of(one) + value_of(two));
            int rank = 0;                                      // groups that come before this one
            for (int d = group_lanes; d < kLanes; d += group_lanes) {
                const int other = (lane + d) % kLanes;
                const uint64_t v = __shfl(value, (int)(threadIdx.x & 63) - lane + other, 64);
                rank += v > value || (v == value && other / group_lanes < group);
            }
            if (rank >= a.group_limit)
#pragma unroll
                for (int i = 0; i < kItems; ++i) key[i] = 0;
        }
        // The k best, one after the other.
        int chosen = -1;
        for (int n = 0; n < a.k; ++n) {
            uint64_t best = 0;
            int expert = INT32_MAX;
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (key[i] > best) { best = key[i]; expert = part.expert(i); }
            for (int d = 1; d < kLanes; d <<= 1) {
                const uint64_t o = __shfl_xor(best, d, 64);
                const int e = __shfl_xor(expert, d, 64);
                if (o > best || (o == best && e < expert)) { best = o; expert = e; }
            }
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (part.mine(i) && part.expert(i) == expert) key[i] = 0;
            if (best != 0 && lane == n) chosen = expert;
        }
        // gates
        const float v = chosen >= 0 ? (float)row[chosen] : -INFINITY;
        float gate = 0.0f;
        if (a.renormalise) {
            const float m = group_max<kLanes>(a.score == P2_SOFTMAX ? v : fminf(v, 0.0f));
            float w = a.score == P2_SOFTMAX ? expf(v - m) : expf(fminf(v, 0.0f) - m) / (1.0f + expf(-fabsf(v)));
            if (chosen < 0) w = 0.0f;
            gate = w / group_sum<kLanes>(w) * a.scale;
            if (inv != inv) gate = (float)inv;                 // (a softmax over something that is not finite)
        } else {
            gate = (a.score == P2_SOFTMAX ? (float)(exp((double)v - most) * inv) : 1.0f / (1.0f + expf(-v))) * a.scale;
        }
        if (there && lane < a.k) {
            a.expert[t * a.k + lane] = chosen;
            a.gate[t * a.k + lane] = chosen >= 0 ? gate : 0.0f;
            if (chosen >= 0) atomicAdd(&count[chosen], 1);
        }
        if (on && lane == 0) atomicAdd(&count[a.experts], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= a.experts; e += kBlock) {
        if (gridDim.x > 1) a.part_count[(int64_t)blockIdx.x * (a.experts + 1) + e] = count[e];
        else if (e < a.experts) a.counts[e] = count[e];
        else a.kept[0] = count[e];
    }
}

// Adds up the blocks' lines: 16 experts a block (the tokens that count are one more column), 16 threads each.
__global__ __launch_bounds__(kBlock) void k_route_sum(RouteForward a, int32_t lines) {
    __shared__ int64_t part[16][16];
    const int x = threadIdx.x % 16, r = threadIdx.x / 16;
    const int e = blockIdx.x * 16 + x;
    int64_t n = 0;
    if (e <= a.experts)
#pragma unroll 8
        for (int l = r; l < lines; l += 16) n += a.part_count[(int64_t)l * (a.experts + 1) + e];
    part[r][x] = n;
    __syncthreads();
    if (r > 0 || e > a.experts) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) n += part[i][x];
    if (e < a.experts) a.counts[e] = n;
    else a.kept[0] = n;
}

// The gradient.  Only the chosen experts' logits have one, but for a softmax that is not renormalised.  A token's row is put together in LDS.
template <typename T> __global__ __launch_bounds__(64) void k_route_backward(RouteBackward a) {
    __shared__ float row[P2_MAX_EXPERTS];
    const int lane = threadIdx.x;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const T* logits = static_cast<const T*>(a.logits) + t * a.stride;
        for (int e = lane; e < a.experts; e += 64) row[e] = 0.0f;
        int expert = lane < a.k ? a.expert[t * a.k + lane] : -1;
        if ((uint32_t)expert >= (uint32_t)a.experts) expert = -1;
        const bool valid = expert >= 0;
        const bool on = __any(valid);
        const float z = valid ? (float)logits[expert] : -INFINITY;
        float d = valid ? a.dgate[t * a.k + lane] * a.scale : 0.0f;
        T* out = static_cast<T*>(a.dlogits) + t * a.dlogits_stride;
        __syncthreads();
        if (a.score == P2_SOFTMAX && !a.renormalise) {
            float m = -INFINITY, s = 0.0f;
            for (int e = lane; e < a.experts; e += 64) m = fmaxf(m, (float)logits[e]);
            m = group_max<64>(m);
            for (int e = lane; e < a.experts; e += 64) s += expf((float)logits[e] - m);
            s = group_sum<64>(s);
            if (valid) atomicAdd(&row[expert], d);
            const float dot = group_sum<64>(valid ? expf(z - m) / s * d : 0.0f);
            __syncthreads();
            for (int e = lane; e < a.experts; e += 64) {
                const float p = expf((float)logits[e] - m) / s;
                out[e] = (T)(on ? p * (row[e] - dot) : 0.0f);
            }
        } else {
            float w = 1.0f, slope = 1.0f;
            if (a.score == P2_SIGMOID) {
                const float far = expf(-fabsf(z)), base = 1.0f / (1.0f + far);
                slope = z > 0.0f ? far * base : base;           // 1 - s
                w = z > 0.0f ? base : far * base;               // s
                if (a.renormalise) {
                    const float m = group_max<64>(fminf(z, 0.0f));
                    w = expf(fminf(z, 0.0f) - m) * base;
                }
            } else {
                w = expf(z - group_max<64>(z));
            }
            if (!valid) w = 0.0f;
            if (a.renormalise && on) {
                w = w / group_sum<64>(w);
                d -= group_sum<64>(w * d);
            }
            if (valid) atomicAdd(&row[expert], w * slope * d);
            __syncthreads();
            for (int e = lane; e < a.experts; e += 64) out[e] = (T)row[e];
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(1024) void k_route_bias(const float* bias, const int64_t* counts, int32_t experts, float rate, float* out) {
    __shared__ int64_t part[16];
    const int e = threadIdx.x;                             // (one thread an expert: 1024 at most)
    const int64_t n = e < experts ? counts[e] : 0;
    int64_t s = over_lanes(n, 64, [](int64_t x, int64_t y) { return x + y; });
    if ((e & 63) == 0) part[e >> 6] = s;
    __syncthreads();
    s = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += part[w];
    // the mean against a count, in whole numbers: sum against experts * count
    const __int128 under = (__int128)s - (__int128)n * experts;
    if (e < experts) out[e] = bias[e] + (under > 0 ? rate : under < 0 ? -rate : 0.0f);
}

int64_t blocks_of(int64_t tokens, const Shape& s) { return std::max<int64_t>(1, std::min(ceil_div(tokens, kBlock / s.lanes), kRouteBlocks)); }

#define P2_ROUTE_CASE(LANES, ITEMS) \
    case LANES * 64 + ITEMS: k_route_forward<T, LANES, ITEMS><<<grid, dim3(kBlock), 0, s>>>(a, shape.group_lanes); break;
#define P2_ROUTE_CASES(ITEMS)                                                                                        \
    P2_ROUTE_CASE(1, ITEMS) P2_ROUTE_CASE(2, ITEMS) P2_ROUTE_CASE(4, ITEMS) P2_ROUTE_CASE(8, ITEMS) P2_ROUTE_CASE(16, ITEMS) \
    P2_ROUTE_CASE(32, ITEMS) P2_ROUTE_CASE(64, ITEMS)

template <typename T> void route(const RouteForward& a, const Shape& shape, int64_t blocks, hipStream_t s) {
    const dim3 grid((unsigned)blocks);
    switch (shape.lanes * 64 + shape.items) {
        P2_ROUTE_CASES(8)
        P2_ROUTE_CASES(16)
        P2_ROUTE_CASES(32)
    }
}

}  // namespace

int64_t route_forward_blocks(int64_t tokens, int32_t experts, int32_t k, int32_t groups) { return blocks_of(tokens, shape_of(experts, k, groups)); }

hipError_t launch_route_forward(const RouteForward& a, hipStream_t s) {
    const Shape shape = shape_of(a.experts, a.k, a.groups);
    const int64_t blocks = blocks_of(a.tokens, shape);
    if (a.type == P2_F32) route<float>(a, shape, blocks, s);
    else if (a.type == P2_BF16) route<bf16_t>(a, shape, blocks, s);
    else route<half_t>(a, shape, blocks, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    k_route_sum<<<dim3((unsigned)ceil_div(a.experts + 1, 16)), dim3(kBlock), 0, s>>>(a, (int32_t)blocks);
    return hipGetLastError();
}

hipError_t launch_route_backward(const RouteBackward& a, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<int64_t>(a.tokens, 8192));
    if (a.type == P2_F32) k_route_backward<float><<<grid, dim3(64), 0, s>>>(a);
    else if (a.type == P2_BF16) k_route_backward<bf16_t><<<grid, dim3(64), 0, s>>>(a);
    else k_route_backward<half_t><<<grid, dim3(64), 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_route_bias(const float* bias, const int64_t* counts, int32_t experts, float rate, float* out, hipStream_t s) {
    k_route_bias<<<dim3(1), dim3(1024), 0, s>>>(bias, counts, experts, rate, out);
    return hipGetLastError();
}

}  // namespace p2
