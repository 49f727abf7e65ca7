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
// As many blocks as the units hold at once: with a bias three a unit (168 registers), without one four (65536 x 256 fp32 31.9 -> 29.8 us; 128 registers with a bias, too: 41 -> 50).
constexpr int64_t kRouteBlocks = 1024, kBiasedBlocks = 768, kBackwardBlocks = 2048;
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

// ------------------------------------------------------------------------------- the choice in 64 bits, for few tokens

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
__device__ __forceinline__ uint64_t larger(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t smaller(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint32_t most_of(uint32_t a, uint32_t b) { return max(a, b); }
__device__ __forceinline__ double over_wavefront(double v, bool sum) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_xor(v, d, 64);
        v = sum ? v + o : fmax(v, o);
    }
    return v;
}

// One token's choice by a whole wavefront, each group with 64 / (groups rounded up to a power of two) lanes.  What the experts are compared by, as ordered
// numbers, is kept in `key`, of which a lane touches its own experts' places alone; the chosen experts go to `slot`.  (A call of its own, so that its 64-bit numbers take no registers from the kernel; arguments one by one, because a reference would put the
// kernel's own into memory.  A token takes some 3 us, so it is latency that counts.)
template <typename T> __device__ __noinline__ void choose_exactly(const T* row, const float* bias, int experts, int k, int score_kind, int groups, int group_lanes, int group_limit,
                                                                  int group_best, uint64_t* key, int* slot) {
    const int lane = threadIdx.x & 63, group = lane / group_lanes, size = experts / groups;
    const int begin = group < groups ? group * size + lane % group_lanes : 0, end = group < groups ? (group + 1) * size : 0;      // of this lane's experts
    const double minus = -__builtin_huge_val();
    double most = minus, sum = 0.0;
    if (score_kind == P2_SOFTMAX) {
        for (int e = begin; e < end; e += group_lanes) most = fmax(most, (double)(float)row[e]);
        most = over_wavefront(most, false);
        for (int e = begin; e < end; e += group_lanes) sum += exp((double)(float)row[e] - most);
        sum = over_wavefront(sum, true);
    }
    const auto score = [&](double z) { return score_kind == P2_SOFTMAX ? exp(z - most) / sum : 1.0 / (1.0 + exp(-z)); };
    uint64_t one = 0, two = 0;                                 // this lane's largest
    int first = 0, second = 0;
#pragma unroll 4
    for (int e = begin; e < end; e += group_lanes) {
        const double z = (double)(float)row[e];
        const float b = bias ? bias[e] : 0.0f;
        const uint64_t x = z == minus || b == -INFINITY ? 0 : ordered(score(z) + (double)b);
        key[e] = x;
        if (x > one) { two = one; second = first; one = x; first = e; }
        else if (x > two) { two = x; second = e; }
    }
    if (groups > 1) {
        uint64_t top = one, next = two;                        // the group's
        for (int d = 1; d < group_lanes; d <<= 1) {
            const uint64_t o = __shfl_xor(top, d, 64), w = __shfl_xor(next, d, 64);
            next = larger(larger(next, w), smaller(top, o));
            top = larger(top, o);
        }
        uint64_t value = top;
        if (group_best == 2 && top != 0 && next != 0) value = ordered(value_of(top) + value_of(next));
        int rank = 0;                                          // groups that come before this one
        for (int g = 0; g < groups; ++g) {
            const uint64_t v = __shfl(value, g * group_lanes, 64);
            rank += v > value || (v == value && g < group);
        }
        if (rank >= group_limit) {
            for (int e = begin; e < end; e += group_lanes) key[e] = 0;
            one = 0;
        }
    }
    // the largest, by the upper halves, and where they are equal the lower ones, the index (a reduction of 32 bits takes 8 instructions, one of 64 some 40)
    bool known = true;                                         // whether `two` is the lane's next
    for (int n = 0; n < k; ++n) {
        const uint32_t high = group_reduce<64>((uint32_t)(one >> 32), most_of);
        bool best = (uint32_t)(one >> 32) == high;
        const uint64_t whose = __ballot(best);
        uint32_t expert;
        if (whose & (whose - 1)) {
            const uint32_t low = group_reduce<64>(best ? (uint32_t)one : 0u, most_of);
            best = one == ((uint64_t)high << 32 | low);
            expert = ~group_reduce<64>(best ? ~(uint32_t)first : 0u, most_of);
        } else {
            expert = (uint32_t)__builtin_amdgcn_readlane(first, __builtin_ctzll(whose));
        }
        if (lane == 0) slot[n] = high != 0 ? (int)expert : -1;
        if (high != 0 && best && (uint32_t)first == expert) {
            key[first] = 0;
            if (!known) {
                two = 0;
#pragma unroll 4
                for (int e = begin; e < end; e += group_lanes)
                    if (key[e] > two) { two = key[e]; second = e; }
            }
            one = two;
            first = second;
            known = false;
        }
    }
    wavefront_exchange();
}

// ----------------------------------------------------------------------------------------- the choice in 32 bits, for all

// What a token's experts are compared by is a whole number of 32 bits, of which the lowest say which of a lane's values it is: sorting takes an instruction a
// place in the list, and a reduction over lanes one a step.  0: not on offer.
//  - With a bias it is the bits of score + bias + 1 + the largest bias, which is 1 or more: whole numbers are in the order of such floats, and one step of
//    them is 2^-23 at least.
//  - Without one it is the logit's bits in their order, which is that of the scores but where two logits have one score in 64 bits (one_score).
// What the lowest bits and the 32 bits leave open is found out by the gaps: where two neighbours among the k + 1 best, or the last group taken and the
// first one left, are nearer to each other than they may be off, or where something is not finite, or a lane has no more of its list, the token is chosen for
// again in 64 bits.  16-bit logits without a bias need no gaps: they leave 13 bits for the whole index.
__device__ __forceinline__ uint32_t in_order(float f) {
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float out_of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// The logit of a number whose lowest bits (`taken`) say something else.  16-bit logits have zeros there, a negative one's number has ones: it is that logit itself.  32-bit ones come out less by up to
// `taken` steps.
template <bool kExact> __device__ __forceinline__ float logit_of(uint32_t o, uint32_t taken) {
    return out_of_order(kExact && !(o & 0x80000000u) ? o | taken : o & ~taken);
}

// Whether a logit and a smaller one next to it in the order may have one score, or scores that 64 bits round off to the wrong order.  Logits differ by 2^-24 of the larger one at least, scores
// of normal size by some 2^-52 once they are rounded, so that has to do with
//  - sigmoids next to 1: at 16 a step of a logit moves them by 2^-42 (`smaller` is asked about); below -700 they come near what 64 bits hold (`larger` is);
//  - exponentials that far below the row's largest, `most` (0 for sigmoids);
//  - logits next to 0, where those up to 2^-16 may differ by any little: both are asked about.  (Two zeros are one logit, but what comes after them is asked about, too.)
// (Asking takes 3 to 8 % of a choice without a bias: 65536 x 256 fp32 28.4 -> 29.6 us, in four groups of which two 31.5 -> 33.4; at most 12 %, 131072 x 128 bf16 30.1 -> 33.8.)
constexpr float kNextToOne = 16.0f, kNextToNothing = -700.0f, kNextToZero = 0x1p-16f;
__device__ __forceinline__ bool little(float z) { return fabsf(z) < kNextToZero && z != 0.0f; }
__device__ __forceinline__ bool one_score(int32_t score, float larger, float smaller, float most) {
    return larger - most < kNextToNothing || (score == P2_SIGMOID && smaller > kNextToOne) || little(larger) || little(smaller);
}
// Whether that has to be asked at all: of the larger one.
__device__ __forceinline__ bool far_out(int32_t score, float z, float most) {
    return z - most < kNextToNothing || z > (score == P2_SIGMOID ? kNextToOne : INFINITY) || fabsf(z) < kNextToZero;
}

// The same number, which the compiler takes for a new one: tests of its bits are not made ahead of a loop, where they would take two scalar registers each.
__device__ __forceinline__ uint32_t opaque(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(v));
#endif
    return v;
}

// A lane's kDepth largest, in falling order.
template <int kDepth> struct List {
    uint32_t v[kDepth] = {};
    // the n-th value to come, among the first kFirst: at most n are there
    template <int kFirst> __device__ __forceinline__ void insert(uint32_t x, int n) {
#pragma unroll
        for (int i = kFirst - 1; i > 0; --i)
            if (i <= n) v[i] = max(min(v[i - 1], v[i]), min(max(v[i - 1], v[i]), x));
        v[0] = max(v[0], x);
    }
    __device__ __forceinline__ void pop(bool now) {
#pragma unroll
        for (int i = 0; i + 1 < kDepth; ++i) v[i] = now ? v[i + 1] : v[i];
        v[kDepth - 1] = now ? 0u : v[kDepth - 1];
    }
};

// A lane's values of its group's part of a row, in whole vectors that are asked for without a condition: where the group's end cuts a vector, or lies before
// it, the group's last V values are taken instead, of which those before the lane's place are another lane's.  Groups shorter than a vector are read value by value.
template <typename T, int kItems> struct Part {
    static constexpr int V = 16 / sizeof(T);
    int first, size, lane, lanes;              // the group's first expert and their number; this lane's place in it
    bool there;                                // whether there is such a group (if not, the values are another one's)
    vec_t<T, V> raw[kItems / V];
    __device__ __forceinline__ int at(int i) const { return ((i / V) * lanes + lane) * V; }
    __device__ __forceinline__ int place(int i) const { return size < V ? at(i) + i % V : min(at(i), size - V) + i % V; }
    __device__ __forceinline__ bool mine(int i) const { return there && place(i) >= at(i) && place(i) < size; }
    __device__ __forceinline__ void load(const T* row) {
        if (size >= V) {
#pragma unroll
            for (int q = 0; q < kItems / V; ++q) raw[q] = *reinterpret_cast<const vec_t<T, V>*>(row + first + min(at(q * V), size - V));
        } else {
#pragma unroll
            for (int q = 0; q < kItems / V; ++q)
#pragma unroll
                for (int j = 0; j < V; ++j) raw[q][j] = row[first + min(at(q * V) + j, size - 1)];
        }
    }
};

// How many of the other lanes of 16 have a larger value, of those that lie a multiple of `each` away.
template <int kTurn> __device__ __forceinline__ void turned(uint32_t v, int each, int& larger_ones) {
    if constexpr (kTurn < 16) {
        if ((kTurn & (each - 1)) == 0) larger_ones += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + kTurn, 0xf, 0xf, true) > v;
        turned<kTurn + 1>(v, each, larger_ones);
    }
}

// Lane i's gate from the i-th choice and its logit v; most and inv: the softmax's largest logit and the inverse of its sum.  (expf, which unlike the instruction gives
// numbers below 2^-126, too.)
template <int kLanes> __device__ __forceinline__ float gate_of(const RouteForward& a, int chosen, float v, float most, float inv) {
    float gate;
    if (a.score == P2_SOFTMAX) {
        if (!a.renormalise) return expf(v - most) * inv;
        const float m = group_max<kLanes>(v);                  // (by all lanes, whether chosen or not)
        gate = chosen >= 0 ? expf(v - m) : 0.0f;
        gate = gate * __builtin_amdgcn_rcpf(group_sum<kLanes>(gate));
        return inv != inv ? inv : gate;                        // (a softmax over something that is not finite)
    }
    // sigmoid(z) = e^min(z, 0) / (1 + e^-|z|), and of all of them by the largest min(z, 0), so that tiny ones keep their digits
    const float base = __builtin_amdgcn_rcpf(1.0f + expf(-fabsf(v))), under = fminf(v, 0.0f);
    const float m = a.renormalise ? group_max<kLanes>(chosen >= 0 ? under : -INFINITY) : 0.0f;
    gate = chosen >= 0 ? expf(under - m) * base : 0.0f;
    if (v != v) gate = v;
    return a.renormalise ? gate * __builtin_amdgcn_rcpf(group_sum<kLanes>(gate)) : gate;
}

// Bound by its vector instructions: 65536 tokens over 256 experts in eight groups, eight each, 35 us (fp32, sigmoid, bias): some 190 a token and lane, whose issue takes 66 % of the units' busy cycles; the
// logits alone would take 14.  Few, wide lanes a token: every reduction over lanes is DPP, and a lane's sorted list saves k passes over its values.  Blocks take tokens in turn, the next
// one's logits under way.
// A list of kDepth is spent where a lane has to give up that many, which for k of 6 and more is common with few lanes in the groups that are open: 65536 tokens over 256 experts in 16 groups, eight each, 40 us
// with four groups open and 232 with one, where every token is chosen for again.
// kAlone: one block has all tokens, and chooses in 64 bits itself; else such tokens are marked for the next kernel.
template <typename T, int kLanes, int kItems, bool kBiased, bool kAlone> __global__ __launch_bounds__(kBlock, kBiased || kAlone || kItems > 16 ? 2 : 4) void k_route_forward(RouteForward a, int32_t group_lanes) {
    typedef Part<T, kItems> P;
    constexpr int kTokens = kBlock / kLanes, kInWave = 64 / kLanes;
    constexpr int kDepth = 6;
    constexpr bool kExact = !kBiased && sizeof(T) == 2;        // numbers that differ, in the order of the choice
    constexpr uint32_t kMask = kExact ? 0x3ff : kItems - 1;
    extern __shared__ uint64_t keys[];                         // kAlone: [wavefronts][experts]
    __shared__ int32_t count[P2_MAX_EXPERTS + 1];
    __shared__ int slots[kTokens][kLanes + 1];                 // (the last one: what is no choice)
    __shared__ float sizes[kBlock / 64];
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e <= a.experts; e += kBlock) count[e] = 0;
    const int group_shift = __builtin_ctz((uint32_t)group_lanes), group = lane >> group_shift;
    P part;
    part.size = a.experts / a.groups;
    part.there = group < a.groups;
    part.first = part.there ? group * part.size : 0;
    part.lane = lane & (group_lanes - 1);
    part.lanes = group_lanes;
    // What a score may be off by: its exponential's argument, the instructions, and of a softmax the sum.
    const float off = a.score == P2_SOFTMAX ? (kItems + 16) * 0x1p-24f : 3e-7f;
    float bias[kBiased ? kItems : 1] = {}, largest = 0.0f;
    uint32_t own = 0, offer = 0;                               // of this lane's values: its own to count, and those on offer by their bias
#pragma unroll
    for (int i = 0; i < kItems; ++i) own |= (uint32_t)part.mine(i) << i;
    offer = own;
    if constexpr (kBiased) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            bias[i] = a.bias[part.first + min(part.place(i), part.size - 1)];
            if (bias[i] == -INFINITY) offer &= ~(1u << i);
            else largest = bias[i] == bias[i] ? fmaxf(largest, fabsf(bias[i])) : INFINITY;
        }
        largest = group_max<64>(largest);
        if ((threadIdx.x & 63) == 0) sizes[wave] = largest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kBlock / 64; ++w) largest = fmaxf(largest, sizes[w]);
#pragma unroll
        for (int i = 0; i < kItems; ++i) bias[i] += 1.0f + largest;
    }
    const bool all_on_offer = __all(offer == (uint32_t)((uint64_t(1) << kItems) - 1));
    // How many steps two neighbours have to be apart, and two groups' values: twice what they are off by, and what the lowest bits take.  (Biases so large, infinite or
    // unordered leave all tokens to 64 bits; a logit is off by its lowest bits alone.)
    const bool large = !(largest < 1e3f);
    const float roundings = (kItems + 6) * (2.0f + 2.0f * largest);
    const uint32_t apart = kExact ? 0 : kBiased ? (uint32_t)(large ? 0.0f : 2.0f * off * 0x1p23f + roundings) : 2 * kItems + 4;
    const float apart_sum = 4.0f * off + 2e-6f + 0x1p-23f * (2.0f * roundings + kLanes * (6.0f + 4.0f * largest));
    if (!kAlone && blockIdx.x == 0)                            // (the next kernel adds to them)
        for (int e = threadIdx.x; e <= a.experts; e += kBlock) *(e < a.experts ? &a.counts[e] : a.kept) = 0;
    const int64_t stride = (int64_t)gridDim.x * kTokens;
    const auto row_of = [&](int64_t t) { return static_cast<const T*>(a.logits) + (t < a.tokens ? t : a.tokens - 1) * a.stride; };
    const int64_t begin = (int64_t)blockIdx.x * kTokens;
    __syncthreads();
    if (begin < a.tokens) part.load(row_of(begin + threadIdx.x / kLanes));
    for (int64_t t0 = begin; t0 < a.tokens; t0 += stride) {
        const int64_t t = t0 + threadIdx.x / kLanes;
        const bool there = t < a.tokens;
        float z[kItems], all = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) z[i] = (float)part.raw[i / P::V][i % P::V];
        if (t0 + stride < a.tokens) part.load(row_of(t + stride));
        bool keep = there && (!a.keep || a.keep[there ? t : 0]), odd = large;
#pragma unroll
        for (int i = 0; i < kItems; ++i) all += z[i];
        const bool special = !all_on_offer || !__all(fabsf(all) < 1e30f);      // not all are ordinary numbers, this lane's own, and on offer
        if (special) {
            bool any = false, bad = false;
            uint32_t own_now = opaque(own);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (!(own_now >> i & 1)) z[i] = -INFINITY;
                any |= z[i] != -INFINITY;
                bad |= !(fabsf(z[i]) < 1e30f) && z[i] != -INFINITY;
            }
            const uint32_t both = group_reduce<kLanes>((uint32_t)any | (uint32_t)bad << 1, [](uint32_t x, uint32_t y) { return x | y; });
            keep = keep && (both & 1);
            odd |= (both & 2) != 0;
        }
        // the scores, in 32 bits
        float most = 0.0f, inv = 1.0f;
        uint32_t key[kItems];
        if (a.score == P2_SOFTMAX) {
            float e[kItems], s = 0.0f;
            most = z[0];
#pragma unroll
            for (int i = 1; i < kItems; ++i) most = fmaxf(most, z[i]);
            most = group_max<kLanes>(most);
#pragma unroll
            for (int i = 0; i < kItems; ++i) { e[i] = __builtin_amdgcn_exp2f((z[i] - most) * kLog2e); s += e[i]; }
            s = group_sum<kLanes>(s);
            inv = __builtin_amdgcn_rcpf(s);
            if constexpr (kBiased)
#pragma unroll
                for (int i = 0; i < kItems; ++i) key[i] = __float_as_uint(fmaf(e[i], inv, bias[i]));
        } else if constexpr (kBiased) {
#pragma unroll
            for (int i = 0; i < kItems; ++i) key[i] = __float_as_uint(__builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z[i] * -kLog2e)) + bias[i]);
        }
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            if constexpr (!kBiased) key[i] = in_order(z[i]);
            key[i] = (key[i] & ~kMask) | (kExact ? kMask - (uint32_t)(part.first + part.place(i)) : kMask - i);
        }
        if (special) {
            const uint32_t offer_now = opaque(offer);
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (z[i] == -INFINITY || !(offer_now >> i & 1)) key[i] = 0;
        }
        List<kDepth> list;
        if (a.k <= 2) {
#pragma unroll
            for (int i = 0; i < kItems; ++i) list.template insert<3>(key[i], i);
        } else {
#pragma unroll
            for (int i = 0; i < kItems; ++i) list.template insert<kDepth>(key[i], i);
        }
        // groups
        if (a.groups > 1) {
            uint32_t one = list.v[0], two = list.v[1];         // the group's largest
            for (int d = 1; d < group_lanes; d <<= 1) {
                const uint32_t o = __shfl_xor(one, d, 64), w = __shfl_xor(two, d, 64);
                two = max(max(two, w), min(one, o));
                one = max(one, o);
            }
            // its value, as a whole number with the group in the lowest bits
            const uint32_t group_bits = kExact && a.group_best == 1 ? kMask : kLanes - 1;
            uint32_t value = one;
            if (a.group_best == 2) {
                const auto score = [&](uint32_t key) {
                    if constexpr (kBiased) return __uint_as_float(key & ~kMask);
                    const float x = logit_of<kExact>(key, kMask);
                    return a.score == P2_SOFTMAX ? __builtin_amdgcn_exp2f((x - most) * kLog2e) * inv : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -kLog2e));
                };
                // (a group with one on offer has one bias alone: the other's part, which every sum of two has, is added)
                const float sum = (one ? score(one) : 0.0f) + (two ? score(two) : kBiased ? 1.0f + largest : 0.0f);
                value = one ? __float_as_uint(sum + 1.0f) : 0;
            }
            if (value) value = (value & ~group_bits) | (group_bits - group);
            int rank = 0;                                      // groups that come before this one
            if constexpr (kLanes == 16) {
                // (a row of 16 lanes turned by d)
                turned<1>(value, group_lanes, rank);
            } else {
                for (int d = group_lanes; d < kLanes; d += group_lanes)
                    rank += (uint32_t)__shfl((int)value, (int)(threadIdx.x & 63) - lane + ((lane + d) & (kLanes - 1)), 64) > value;
            }
            const bool taken = rank < a.group_limit && value;
            // (without a bias: whether some group's largest is where logits have one score)
            const bool doubt = !kBiased && a.group_best == 1 && __any(far_out(a.score, logit_of<kExact>(value, group_bits), most));
            if (!kExact || a.group_best == 2 || doubt) {
                const uint32_t last = ~group_reduce<kLanes>(taken ? ~value : 0u, most_of), left = group_reduce<kLanes>(taken ? 0u : value, most_of);
                // (a softmax's scores go by differences of logits, of which the lowest bits are off by steps of the logits' size)
                const float size = !kBiased && !kExact && a.score == P2_SOFTMAX ? 4.0f * kItems * 0x1p-23f * fabsf(most) : 0.0f;
                if (a.group_best == 2) odd |= left && !(__uint_as_float(last) - __uint_as_float(left) > apart_sum + size);
                else if (!kExact) odd |= left && last - left <= apart + kLanes;
                if (doubt) {
                    const float taken_last = logit_of<kExact>(last, group_bits), left_first = logit_of<kExact>(left, group_bits);
                    const bool behind = group_reduce<kLanes>((uint32_t)(value && little(logit_of<kExact>(value, group_bits))), most_of) != 0;
                    odd |= left && (one_score(a.score, taken_last, left_first, most) || (taken_last == 0.0f && left_first == 0.0f && behind));
                }
            }
            if (!taken) list = List<kDepth>();
        }
        // The k best, one after the other: the largest of what the lanes have left.  (One more for the gap after the last.)
        uint32_t best = group_reduce<kLanes>(list.v[0], most_of), gap = ~0u;
        int pops = 0, found = 0;
        for (int n = 0; n < a.k; ++n) {
            const bool owner = list.v[0] == best && best != 0;
            slots[threadIdx.x / kLanes][owner ? n : kLanes] = (int)(kExact ? kMask - (best & kMask) : (best & kMask) | lane << 8);
            found += best != 0;
            pops += owner;
            list.pop(owner);
            const uint32_t next = group_reduce<kLanes>(list.v[0], most_of);
            gap = min(gap, best + ~next);                      // (less 1, so that nothing after nothing is no gap; equal ones have two owners)
            best = next;
        }
        odd |= group_reduce<kLanes>((uint32_t)(pops >= (a.k <= 2 ? 3 : kDepth)), most_of) != 0;
        bool near = false;
        if constexpr (!kExact) {
            const int owners = (int)group_reduce<kLanes>((uint32_t)pops, [](uint32_t x, uint32_t y) { return x + y; });
            odd |= owners != found;
            near = gap <= apart;
        }
        odd = odd && keep;
        near = near && keep && !odd;
        // which value of which lane a slot says (a candidate's number: its lane, and its lowest bits)
        const auto expert_of = [&](int c) {
            if constexpr (kExact) return c;
            const int i = (int)(kMask - (c & kMask)), from = c >> 8;
            const int at = ((i / P::V) * group_lanes + (from & (group_lanes - 1))) * P::V;
            return (from >> group_shift) * part.size + (part.size < P::V ? at : min(at, part.size - P::V)) + i % P::V;
        };
        wavefront_exchange();
        const int my_slot = lane < found ? slots[threadIdx.x / kLanes][lane] : 0;
        int chosen = keep && lane < found ? expert_of(my_slot) : -1;
        const int at_first = chosen;
        float logit = -INFINITY;
        if constexpr (!kBiased) {
            if (chosen >= 0) logit = (float)row_of(t)[chosen];
            if (__any(chosen >= 0 && far_out(a.score, logit, most))) {
                const float after = logit_of<kExact>(best, kMask);
                bool doubt = chosen >= 0 && one_score(a.score, logit, lane > 0 ? logit : after, most);
                const bool zeros = chosen >= 0 && logit == 0.0f && after == 0.0f;      // (behind which there may be logits next to 0)
                if (__any(zeros)) {
                    const T* row = row_of(t);
                    bool any = false;
                    for (int e = lane; e < a.experts; e += kLanes) any |= little((float)row[e]);
                    const bool some = group_reduce<kLanes>((uint32_t)zeros, most_of) != 0;         // (by all lanes)
                    doubt |= any && some;
                }
                odd = odd || group_reduce<kLanes>((uint32_t)doubt, most_of) != 0;
                near = near && !odd;
            }
        }
        if (!kExact && __any(near)) {
            // The k + 1 best in 64 bits, one a lane, if the next one is far enough from all of them.
            const uint64_t there_next = __ballot(list.v[0] == best && best != 0) >> ((threadIdx.x & 63) - lane) & (~0ull >> (64 - kLanes));
            const int whose = __builtin_ctzll(there_next | 1ull << 63);
            const int low = (int)(best & kMask);
            list.pop(list.v[0] == best && best != 0);
            const uint32_t next = group_reduce<kLanes>(list.v[0], most_of);
            const bool spent = group_reduce<kLanes>((uint32_t)(pops + 1 >= (a.k <= 2 ? 3 : kDepth)), most_of) != 0;       // (a lane's list, perhaps)
            const bool resolved = kLanes > a.k && best + ~next > apart && __popcll(there_next) <= 1 && !spent;
            const int candidate = lane < found ? chosen : lane == a.k && best != 0 && found == a.k ? expert_of(low | whose << 8) : -1;
            uint64_t v = 0;
            double sum = 1.0;
            const double top = (double)most;
            if (kBiased && a.score == P2_SOFTMAX) {
                sum = 0.0;
                const T* row = row_of(t);
#pragma unroll 1
                for (int e = lane; e < a.experts; e += kLanes) sum += exp((double)(float)row[e] - top);
#pragma unroll
                for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d, 64);
            }
            if (candidate >= 0) {
                const double x = (double)(float)row_of(t)[candidate];
                if constexpr (!kBiased) v = ordered(x);
                else v = ordered((a.score == P2_SOFTMAX ? exp(x - top) / sum : 1.0 / (1.0 + exp(-x))) + (double)a.bias[candidate]);
            }
            int rank = 0;
            for (int n = 0; n <= a.k && n < kLanes; ++n) {
                const int from = (int)(threadIdx.x & 63) - lane + n;
                const uint64_t o = __shfl(v, from, 64);
                const int e = __shfl(candidate, from, 64);
                rank += o > v || (o == v && e < candidate);
            }
            // (those without a candidate take no place)
            if (near && candidate >= 0 && rank < a.k) slots[threadIdx.x / kLanes][rank] = candidate;
            wavefront_exchange();
            if (near) {
                if (resolved) chosen = lane < found ? slots[threadIdx.x / kLanes][lane] : -1;
                else odd = true;
            }
        }
        if constexpr (kAlone) {
            const int exact_lanes = 64 / (kLanes >> group_shift);              // of a group, where a wavefront has one token
            uint64_t again = __ballot(odd && lane == 0);
            while (again) {
                const int leader = __builtin_ctzll(again);
                again &= again - 1;
                const int token = wave * kInWave + leader / kLanes;
                choose_exactly<T>(row_of(t0 + token), a.bias, a.experts, a.k, a.score, a.groups, exact_lanes, a.group_limit, a.group_best, keys + wave * a.experts, slots[token]);
                if ((int)(threadIdx.x & 63) / kLanes == leader / kLanes) chosen = lane < a.k ? slots[token][lane] : -1;
            }
        } else {
            if (lane == 0 && there) a.again[t] = odd;
        }
        if (kBiased || chosen != at_first) logit = chosen >= 0 ? (float)row_of(t)[chosen] : -INFINITY;
        const float gate = gate_of<kLanes>(a, chosen, logit, most, inv);
        if (there && lane < a.k) {
            a.expert[t * a.k + lane] = chosen;
            a.gate[t * a.k + lane] = chosen >= 0 ? gate * a.scale : 0.0f;
            if (chosen >= 0 && (kAlone || !odd)) atomicAdd(&count[chosen], 1);
        }
        if (keep && lane == 0) atomicAdd(&count[a.experts], 1);
        wavefront_exchange();                                  // (the slots have been read)
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= a.experts; e += kBlock) {
        if (!kAlone) a.part_count[(int64_t)blockIdx.x * (a.experts + 1) + e] = count[e];
        else if (e < a.experts) a.counts[e] = count[e];
        else a.kept[0] = count[e];
    }
}

// What is left after the first kernel.  The first blocks add up its lines: four experts each (the tokens that count are one more column), 64 threads an expert.  The
// others choose in 64 bits for the tokens that it has marked, a wavefront each.  Both add whole numbers to counts, in whatever order.  (A launch and a token's 3 us: 8.8 us after 65536 tokens,
// 6.4 after 10007.)
template <typename T> __global__ __launch_bounds__(kBlock) void k_route_finish(RouteForward a, int32_t lines, int32_t sum_blocks, int32_t exact_lanes) {
    extern __shared__ uint64_t keys[];                         // [wavefronts][experts]
    __shared__ int64_t part[kBlock / 4][4];
    __shared__ int slots[kBlock / 64][P2_MAX_CHOSEN];
    if ((int)blockIdx.x < sum_blocks) {
        const int x = threadIdx.x % 4, r = threadIdx.x / 4;
        const int e = blockIdx.x * 4 + x;
        int64_t n = 0;
        if (e <= a.experts)
            for (int l0 = r; l0 < lines; l0 += 6 * (kBlock / 4)) {                     // (six lines under way)
                int32_t v[6];
#pragma unroll
                for (int u = 0; u < 6; ++u) {
                    const int l = l0 + u * (kBlock / 4);
                    v[u] = a.part_count[(int64_t)min(l, lines - 1) * (a.experts + 1) + e];
                    if (l >= lines) v[u] = 0;
                }
#pragma unroll
                for (int u = 0; u < 6; ++u) n += v[u];
            }
        part[r][x] = n;
        __syncthreads();
        if (r >= 4) return;
#pragma unroll
        for (int i = r + 4; i < kBlock / 4; i += 4) n += part[i][x];
        n += __shfl_xor(n, 4, 64);                             // (lanes 4 r + x)
        n += __shfl_xor(n, 8, 64);
        if (r > 0 || e > a.experts) return;
        atomicAdd(reinterpret_cast<unsigned long long*>(e < a.experts ? &a.counts[e] : a.kept), (unsigned long long)n);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t t0 = (int64_t)(blockIdx.x - sum_blocks) * 64; t0 < a.tokens; t0 += (int64_t)(gridDim.x - sum_blocks) * 64) {
        uint64_t again = __ballot(t0 + lane < a.tokens && a.again[min(t0 + lane, a.tokens - 1)]);
        for (int n = 0; again; ++n) {                          // (the block's wavefronts take them in turn)
            const int64_t t = t0 + __builtin_ctzll(again);
            again &= again - 1;
            if (n % (kBlock / 64) != wave) continue;
            const T* row = static_cast<const T*>(a.logits) + t * a.stride;
            choose_exactly<T>(row, a.bias, a.experts, a.k, a.score, a.groups, exact_lanes, a.group_limit, a.group_best, keys + wave * a.experts, slots[wave]);
            float most = -INFINITY, inv = 1.0f;
            if (a.score == P2_SOFTMAX) {
                float s = 0.0f;
                for (int e = lane; e < a.experts; e += 64) most = fmaxf(most, (float)row[e]);
                most = group_max<64>(most);
                for (int e = lane; e < a.experts; e += 64) s += expf((float)row[e] - most);
                inv = 1.0f / group_sum<64>(s);
            }
            const int chosen = lane < a.k ? slots[wave][lane] : -1;
            const float gate = gate_of<64>(a, chosen, chosen >= 0 ? (float)row[chosen] : -INFINITY, most, inv);
            if (lane < a.k) {
                a.expert[t * a.k + lane] = chosen;
                a.gate[t * a.k + lane] = chosen >= 0 ? gate * a.scale : 0.0f;
                if (chosen >= 0) atomicAdd(reinterpret_cast<unsigned long long*>(&a.counts[chosen]), 1ull);
            }
            wavefront_exchange();                              // (the slots have been read)
        }
    }
}

// The gradient.  But for a softmax that is not renormalised only the chosen experts' logits have one, and only these are read.  The choices' parts go to their
// experts' places in a row of LDS of the token's lanes, which holds zeros otherwise and is cleared again after use; only the token's own lanes, which are of one
// wavefront, touch that row.  (Where a token names an expert more than once its parts are added by one instruction, in the order of the lanes.)
// Bound by memory: 65536 tokens over 256 experts, eight each, 21 us for 67 MB written and 39 MB of whole lines around the chosen logits, 5.0 TB/s.
template <typename T, int kLanes, int kItems> __global__ __launch_bounds__(kBlock) void k_route_backward(RouteBackward a, int32_t pitch) {
    typedef Part<T, kItems> P;
    constexpr int kTokens = kBlock / kLanes;
    extern __shared__ float rows[];                            // [kTokens][pitch]
    const int lane = threadIdx.x % kLanes;
    float* slots = rows + threadIdx.x / kLanes * pitch;
    P part;
    part.first = 0;
    part.size = a.experts;
    part.lane = lane;
    part.lanes = kLanes;
    part.there = true;
    const bool dense = a.score == P2_SOFTMAX && !a.renormalise;
    for (int e = lane; e < a.experts; e += kLanes) slots[e] = 0.0f;
    wavefront_exchange();
    const int64_t stride = (int64_t)gridDim.x * kTokens;
    // A token's choices, and the row where it is needed, are asked for while the one before it is worked on.
    int next_expert = -1;
    float next_dgate = 0.0f, next_z = 0.0f;
    const auto row_of = [&](int64_t t) { return static_cast<const T*>(a.logits) + t * a.stride; };
    const auto ask = [&](int64_t t) {
        const int64_t at = min(t, a.tokens - 1) * a.k + min(lane, a.k - 1);
        const int e = a.expert[at];
        next_expert = lane < a.k && (uint32_t)e < (uint32_t)a.experts ? e : -1;
        next_dgate = a.dgate[at];
        if (dense) part.load(row_of(min(t, a.tokens - 1)));
    };
    const auto ask_logit = [&](int64_t t) { next_z = (float)row_of(min(t, a.tokens - 1))[max(next_expert, 0)]; };
    const int64_t start = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes;
    if (start - threadIdx.x / kLanes >= a.tokens) return;
    ask(start);
    ask_logit(start);
    for (int64_t t0 = start - threadIdx.x / kLanes; t0 < a.tokens; t0 += stride) {
        const int64_t t = t0 + threadIdx.x / kLanes;
        const int expert = next_expert;
        const bool valid = expert >= 0;
        const float z = valid ? next_z : -INFINITY;
        float d = valid ? next_dgate * a.scale : 0.0f;
        float o[kItems];
        if (dense)
#pragma unroll
            for (int i = 0; i < kItems; ++i) o[i] = (float)part.raw[i / P::V][i % P::V];
        if (t0 + stride < a.tokens) ask(t + stride);
        float dot = 0.0f, add = d;
        if (dense) {
            // e^(v - m) as 2^(v log2e - m log2e): what the rounding of the second product is off by is common to the row
            float m = o[0], s = 0.0f;
#pragma unroll
            for (int i = 1; i < kItems; ++i) m = fmaxf(m, o[i]);
            m = group_max<kLanes>(m);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                o[i] = __builtin_amdgcn_exp2f((o[i] - m) * kLog2e);
                s += part.mine(i) ? o[i] : 0.0f;
            }
            const float inv = 1.0f / group_sum<kLanes>(s);
#pragma unroll
            for (int i = 0; i < kItems; ++i) o[i] *= inv;
            dot = group_sum<kLanes>(valid ? __builtin_amdgcn_exp2f((z - m) * kLog2e) * inv * d : 0.0f);
        } else {
            float w = 1.0f, slope = 1.0f;
            const float far = expf(-fabsf(z)), base = __builtin_amdgcn_rcpf(1.0f + far);
            if (a.score == P2_SIGMOID) {
                slope = z > 0.0f ? far * base : base;          // 1 - s
                w = z > 0.0f ? base : far * base;              // s
            }
            if (a.renormalise) {
                const float under = a.score == P2_SIGMOID ? fminf(z, 0.0f) : z, m = group_max<kLanes>(under);
                w = valid ? expf(under - m) * (a.score == P2_SIGMOID ? base : 1.0f) : 0.0f;
                const float sum = group_sum<kLanes>(w);
                w = w / (sum == 0.0f ? 1.0f : sum);            // (no choices: 0)
                d -= group_sum<kLanes>(w * d);
            }
            add = w * slope * d;
        }
        if (valid) atomicAdd(&slots[expert], add);
        wavefront_exchange();
        const bool on = group_reduce<kLanes>((uint32_t)valid, most_of) != 0;
        if (t0 + stride < a.tokens) ask_logit(t + stride);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const float u = slots[min(part.place(i), a.experts - 1)];
            o[i] = dense ? (on ? o[i] * (u - dot) : 0.0f) : u;
        }
        wavefront_exchange();
        if (valid) slots[expert] = 0.0f;
        wavefront_exchange();
        if (t < a.tokens) {
            T* out = static_cast<T*>(a.dlogits) + t * a.dlogits_stride;
#pragma unroll
            for (int q = 0; q < kItems / P::V; ++q) {
                float v[P::V];
#pragma unroll
                for (int j = 0; j < P::V; ++j) v[j] = o[q * P::V + j];
                if (a.experts >= P::V) {
                    if (part.at(q * P::V) < a.experts) store_vec<T, P::V>(out + part.place(q * P::V), v);
                } else {
                    store_part<T, P::V>(out + part.at(q * P::V), a.experts - part.at(q * P::V), v);
                }
            }
        }
    }
}

// One block: a launch's time, 4.1 us behind other work.
__global__ __launch_bounds__(1024) void k_route_bias(const float* bias, const int64_t* counts, int32_t experts, float rate, float* out) {
    __shared__ int64_t part[16];
    const int e = threadIdx.x;                             // (one thread an expert)
    const int64_t n = e < experts ? counts[e] : 0;
    int64_t s = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
    if ((e & 63) == 0) part[e >> 6] = s;
    __syncthreads();
    s = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += part[w];
    // the mean against a count, in whole numbers: sum against experts * count
    const __int128 under = (__int128)s - (__int128)n * experts;
    if (e < experts) out[e] = bias[e] + (under > 0 ? rate : under < 0 ? -rate : 0.0f);
}

size_t key_bytes(int32_t experts) { return (size_t)experts * 8 * (kBlock / 64); }
// (One block takes two rounds of tokens where that saves the second launch and no token is chosen for again one after the other: 32 tokens over 256 experts without a bias 8.2 -> 6.3 us, with one 11.1 -> 11.8.)
int64_t blocks_of(int64_t tokens, const Shape& s, bool biased) {
    const int64_t rounds = std::max<int64_t>(1, ceil_div(tokens, kBlock / s.lanes));
    return !biased && rounds == 2 ? 1 : std::min(rounds, biased ? kBiasedBlocks : kRouteBlocks);
}

#define P2_ROUTE_CASE(LANES, ITEMS)                                                                                               \
    case LANES * 64 + ITEMS:                                                                                                     \
        if (blocks == 1) k_route_forward<T, LANES, ITEMS, kBiased, true><<<grid, dim3(kBlock), room, s>>>(a, shape.group_lanes); \
        else k_route_forward<T, LANES, ITEMS, kBiased, false><<<grid, dim3(kBlock), 0, s>>>(a, shape.group_lanes);               \
        break;

template <typename T, bool kBiased> void route(const RouteForward& a, const Shape& shape, int64_t blocks, hipStream_t s) {
    const dim3 grid((unsigned)blocks);
    const size_t room = key_bytes(a.experts);
    switch (shape.lanes * 64 + shape.items) {                  // (what shape_of gives)
        P2_ROUTE_CASE(1, 8)
        P2_ROUTE_CASE(2, 8)
        P2_ROUTE_CASE(4, 8)
        P2_ROUTE_CASE(8, 8)
        P2_ROUTE_CASE(16, 8)
        P2_ROUTE_CASE(32, 8)
        P2_ROUTE_CASE(64, 8)
        P2_ROUTE_CASE(16, 16)
        P2_ROUTE_CASE(32, 16)
        P2_ROUTE_CASE(64, 16)
        P2_ROUTE_CASE(64, 32)
    }
}
template <typename T> hipError_t route(const RouteForward& a, const Shape& shape, int64_t blocks, hipStream_t s) {
    if (a.bias) route<T, true>(a, shape, blocks, s);
    else route<T, false>(a, shape, blocks, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    const int64_t sums = ceil_div(a.experts + 1, 4), others = std::min<int64_t>(ceil_div(a.tokens, 64), 2048);
    k_route_finish<T><<<dim3((unsigned)(sums + others)), dim3(kBlock), key_bytes(a.experts), s>>>(a, (int32_t)blocks, (int32_t)sums, 64 / (shape.lanes / shape.group_lanes));
    return hipGetLastError();
}

#define P2_ROUTE_BACKWARD_CASE(LANES, ITEMS) \
    case LANES * 64 + ITEMS: k_route_backward<T, LANES, ITEMS><<<grid, dim3(kBlock), room, s>>>(a, pitch); break;
template <typename T> void backward(const RouteBackward& a, const Shape& shape, dim3 grid, size_t room, int32_t pitch, hipStream_t s) {
    switch (shape.lanes * 64 + shape.items) {                  // (what shape_of gives for one group)
        P2_ROUTE_BACKWARD_CASE(1, 8)
        P2_ROUTE_BACKWARD_CASE(2, 8)
        P2_ROUTE_BACKWARD_CASE(4, 8)
        P2_ROUTE_BACKWARD_CASE(8, 8)
        P2_ROUTE_BACKWARD_CASE(16, 8)
        P2_ROUTE_BACKWARD_CASE(32, 8)
        P2_ROUTE_BACKWARD_CASE(64, 8)
        P2_ROUTE_BACKWARD_CASE(16, 16)
        P2_ROUTE_BACKWARD_CASE(32, 16)
        P2_ROUTE_BACKWARD_CASE(64, 16)
    }
}

}  // namespace

int64_t route_forward_blocks(int64_t tokens, int32_t experts, int32_t k, int32_t groups) {
    const Shape s = shape_of(experts, k, groups);
    return std::max(blocks_of(tokens, s, false), blocks_of(tokens, s, true));
}

hipError_t launch_route_forward(const RouteForward& a, hipStream_t s) {
    const Shape shape = shape_of(a.experts, a.k, a.groups);
    const int64_t blocks = blocks_of(a.tokens, shape, a.bias != nullptr);
    return a.type == P2_F32 ? route<float>(a, shape, blocks, s) : a.type == P2_BF16 ? route<bf16_t>(a, shape, blocks, s) : route<half_t>(a, shape, blocks, s);
}

hipError_t launch_route_backward(const RouteBackward& a, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const Shape shape = shape_of(a.experts, a.k, 1);
    const int32_t pitch = a.experts + 4;
    const dim3 grid((unsigned)std::min(ceil_div(a.tokens, kBlock / shape.lanes), kBackwardBlocks));
    const size_t room = (size_t)(kBlock / shape.lanes) * pitch * sizeof(float);
    if (a.type == P2_F32) backward<float>(a, shape, grid, room, pitch, s);
    else if (a.type == P2_BF16) backward<bf16_t>(a, shape, grid, room, pitch, s);
    else backward<half_t>(a, shape, grid, room, pitch, s);
    return hipGetLastError();
}

hipError_t launch_route_bias(const float* bias, const int64_t* counts, int32_t experts, float rate, float* out, hipStream_t s) {
    k_route_bias<<<dim3(1), dim3((unsigned)ceil_div(experts, 64) * 64), 0, s>>>(bias, counts, experts, rate, out);
    return hipGetLastError();
}

}  // namespace p2
