// The router's balance: the k best experts of each token, their probabilities, counts and probability sums per expert,
// the balance loss, and the gradient with respect to the logits.
//
// A token's logits are read once and stay in the registers of kLanes lanes, kItems each (a lane holds whole 16-byte
// vectors); a wavefront takes 64 / kLanes tokens at a time.  Choosing goes by keys in which a larger logit, and of equal ones
// the lower index, is the larger whole number: it is exact and does not depend on how the softmax is rounded.
#include <algorithm>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kBalanceBlock = 512;
constexpr int64_t kBalanceBlocks = 512;                // two blocks a compute unit
constexpr float kLog2e = 1.44269504088896340736f;

// e^(v - m), v and m finite or not; 1 ulp of 2^x and what the product rounds.
__device__ __forceinline__ float exp_of(float v, float m) { return __builtin_amdgcn_exp2f((v - m) * kLog2e); }

// Keys: whole numbers in the order of the logits, and of equal ones in the order of falling indexes.  A float's bits, turned
// over where it is negative, are in its order (NaN aside: with_nan puts it above everything).  16-bit logits leave the lowest 13 of them unused: the index goes there; for 32-bit
// ones it takes 32 bits more.  -0 is 0; what is not above -inf (kNone) is never chosen.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
// Whether it is a NaN's: above +inf's, or below -inf's.
__device__ __forceinline__ bool ordered_nan(uint32_t o) { return o > 0xff800000u || o < 0x007fffffu; }
__device__ __forceinline__ float from_ordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
constexpr uint32_t kNone = 0x007fffffu;                // ordered(-inf)
template <typename T> struct Key {                     // half_t, bf16_t
    typedef uint32_t type;
    static constexpr uint32_t kLow = 0x1fffu;
    static __device__ __forceinline__ type of(float f, int e) { return (ordered(f) & ~kLow) | (kLow - (uint32_t)e); }
    static __device__ __forceinline__ type with_nan(type k) { return ordered_nan(k | kLow) && ordered_nan(k & ~kLow) ? k | ~kLow : k; }
    static __device__ __forceinline__ bool real(type k) { return (k & ~kLow) > (kNone & ~kLow); }
    static __device__ __forceinline__ int index(type k) { return (int)(kLow - (k & kLow)); }
    static __device__ __forceinline__ float value(type k) { return from_ordered(k & 0x80000000u ? k & ~kLow : k | kLow); }
};
template <> struct Key<float> {
    typedef uint64_t type;
    static __device__ __forceinline__ type of(float f, int e) { return (uint64_t)ordered(f) << 32 | (0xffffffffu - (uint32_t)e); }
    static __device__ __forceinline__ type with_nan(type k) { return ordered_nan((uint32_t)(k >> 32)) ? k | 0xffffffff00000000ull : k; }
    static __device__ __forceinline__ bool real(type k) { return (uint32_t)(k >> 32) > kNone; }
    static __device__ __forceinline__ int index(type k) { return (int)(0xffffffffu - (uint32_t)k); }
    static __device__ __forceinline__ float value(type k) { return from_ordered((uint32_t)(k >> 32)); }
};

__device__ __forceinline__ double block_sum(double v, double* buf) {       // thread 0 gets it
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) if (threadIdx.x == 0) v += buf[w];
    return v;
}
__device__ __forceinline__ float loss_of(double sum, int64_t kept, int32_t experts, int32_t k) {
    return kept > 0 ? (float)(sum * experts / ((double)k * (double)kept * (double)kept)) : 0.0f;
}

// This lane's kItems logits of a row, in whole vectors that are asked for without a condition (load_whole); a row shorter than a
// vector, which one lane has alone, value by value.  place(i): the expert that value i belongs to; mine(i): whether it is this
// lane's to count.
template <typename T, int kLanes, int kItems> struct Row {
    static constexpr int V = 16 / sizeof(T);
    static constexpr int kVecs = kItems / V;
    vec_t<T, V> raw[kVecs];
    static __device__ __forceinline__ bool is_short(int experts) { return kLanes == 1 && experts < V; }
    static __device__ __forceinline__ int first(int lane, int q) { return (q * kLanes + lane) * V; }
    static __device__ __forceinline__ int place(int lane, int experts, int i) {
        return is_short(experts) ? i : vec_at(first(lane, i / V), experts, V) + i % V;
    }
    static __device__ __forceinline__ bool mine(int lane, int experts, int i) {
        return is_short(experts) ? i < experts : own<V, false>(first(lane, i / V), experts, i % V);
    }
    // Where expert e's value lies in a row of LDS: the lanes' i-th values side by side.  Rows are kPitch apart, so that what the
    // wavefront's lanes read at once lies in different banks.
    static constexpr int kPitch = kLanes * (kItems + 1);
    static __device__ __forceinline__ int slot(int e) {
        const int v = e / V;
        return ((v / kLanes) * V + e % V) * kLanes + v % kLanes;
    }
    __device__ __forceinline__ void load(const T* row, int lane, int experts) {
        if (!is_short(experts)) {
#pragma unroll
            for (int q = 0; q < kVecs; ++q) raw[q] = load_whole<T, V>(row, first(lane, q), experts);
        } else {
#pragma unroll
            for (int i = 0; i < kItems; ++i) raw[i / V][i % V] = row[min(i, experts - 1)];
        }
    }
    __device__ __forceinline__ void get(float (&p)[kItems]) const {
#pragma unroll
        for (int i = 0; i < kItems; ++i) p[i] = (float)raw[i / V][i % V];
    }
    // `other` in the place of values that are not this lane's to count
    static __device__ __forceinline__ void count_once(int lane, int experts, float other, float (&p)[kItems]) {
        if (kLanes * kItems != experts)                    // (else all of them are)
#pragma unroll
            for (int i = 0; i < kItems; ++i) p[i] = mine(lane, experts, i) ? p[i] : other;
    }
    static __device__ __forceinline__ float sum_once(int lane, int experts, const float (&p)[kItems]) {
        float s = 0.0f;
        if (kLanes * kItems == experts) {
#pragma unroll
            for (int i = 0; i < kItems; ++i) s += p[i];
        } else {
#pragma unroll
            for (int i = 0; i < kItems; ++i) s += mine(lane, experts, i) ? p[i] : 0.0f;
        }
        return s;
    }
    // Every lane stores all of its vectors, also where another one stores the same: with stores that depend on nothing the compiler
    // can count what is under way, and the next row's loads need not wait for them.
    __device__ __forceinline__ static void store(T* row, int lane, int experts, const float (&o)[kItems]) {
#pragma unroll
        for (int q = 0; q < kVecs; ++q) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = o[q * V + j];
            if (!is_short(experts)) store_vec<T, V>(row + vec_at(first(lane, q), experts, V), v);
            else store_part<T, V>(row + q * V, experts - q * V, v);
        }
    }
};

template <typename T, int kLanes, int kItems> __global__ __launch_bounds__(kBalanceBlock, 4) void k_balance_forward(BalanceForward a) {
    typedef typename Key<T>::type K;
    typedef Row<T, kLanes, kItems> R;
    constexpr int kTokens = kBalanceBlock / kLanes;
    constexpr int kWaves = kBalanceBlock / 64;
    constexpr int kWidth = kLanes * kItems;
    __shared__ int32_t count[P2_MAX_EXPERTS + 1];
    __shared__ float sums[kWaves][kWidth];
    __shared__ double buf[kWaves];
    const int lane = threadIdx.x % kLanes;
    for (int e = threadIdx.x; e <= a.experts; e += kBalanceBlock) count[e] = 0;
    __syncthreads();
    float acc[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) acc[i] = 0.0f;
    // A token's logits are asked for while the one before it is worked on.
    const int64_t stride = (int64_t)gridDim.x * kTokens;
    R next;
    bool next_keep = false;
    auto ask = [&](int64_t t) {
        const int64_t at = t < a.tokens ? t : a.tokens - 1;
        next.load(static_cast<const T*>(a.logits) + at * a.stride, lane, a.experts);
        next_keep = t < a.tokens && (!a.keep || a.keep[at]);
    };
    const int64_t first = (int64_t)blockIdx.x * kTokens;
    if (first < a.tokens) ask(first + threadIdx.x / kLanes);
    for (int64_t t0 = first; t0 < a.tokens; t0 += stride) {
        const int64_t t = t0 + threadIdx.x / kLanes;
        const bool there = t < a.tokens, keep = next_keep;
        float p[kItems];
        K key[kItems];
        next.get(p);
        R::count_once(lane, a.experts, -INFINITY, p);
        if (t0 + stride < a.tokens) ask(t + stride);
        float m = p[0];
#pragma unroll
        for (int i = 1; i < kItems; ++i) m = fmaxf(m, p[i]);
        m = group_max<kLanes>(m);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            key[i] = Key<T>::of(p[i], R::place(lane, a.experts, i));
            p[i] = exp_of(p[i], m);
        }
        R::count_once(lane, a.experts, 0.0f, p);           // (m may be -inf)
#pragma unroll
        for (int i = 0; i < kItems; ++i) s += p[i];
        s = group_sum<kLanes>(s);
        if (__any(s != s)) {                               // a NaN, or an infinity: see which, NaN is above everything
#pragma unroll
            for (int i = 0; i < kItems; ++i) key[i] = Key<T>::with_nan(key[i]);
        }
        const float inv = __builtin_amdgcn_rcpf(s);
        // The k best, one after the other: the next is the largest key below the last, and as whole numbers that wrap around
        // key - last is the larger the nearer the key is below.  Lane i % kLanes keeps the i-th until as many as there are lanes
        // are to be written.
        K held = 0, last = 0;
        bool on = false;
        for (int i = 0; i < a.k; ++i) {
            K best = key[0] - last;
#pragma unroll
            for (int q = 1; q < kItems; ++q) { const K d = key[q] - last; best = d > best ? d : best; }
            best = group_reduce<kLanes>(best, [](K x, K y) { return x > y ? x : y; });
            last += best;                                  // (there are k keys at least: -inf has one, too)
            if (i == 0) on = keep && Key<T>::real(last);
            if (i % kLanes == lane) held = last;
            if ((i + 1) % kLanes == 0 || i + 1 == a.k) {
                const int slot = i - i % kLanes + lane;
                if (there && slot <= i) {
                    const bool real = keep && Key<T>::real(held);
                    const int e = Key<T>::index(held);
                    a.expert[t * a.k + slot] = real ? e : -1;
                    a.gate[t * a.k + slot] = real ? exp_of(Key<T>::value(held), m) * inv : 0.0f;
                    if (real) atomicAdd(&count[e], 1);
                }
            }
        }
        if (on) {
            if (lane == 0) atomicAdd(&count[a.experts], 1);
#pragma unroll
            for (int i = 0; i < kItems; ++i) acc[i] += p[i] * inv;
        }
    }
    // lanes of a wavefront that hold the same experts, then the wavefronts, in a fixed order
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
#pragma unroll
        for (int d = kLanes; d < 64; d <<= 1) acc[i] += __shfl_xor(acc[i], d, 64);
        if ((threadIdx.x & 63) < kLanes && R::mine(lane, a.experts, i)) sums[threadIdx.x >> 6][R::place(lane, a.experts, i)] = acc[i];
    }
    __syncthreads();
    const bool alone = gridDim.x == 1;
    double l = 0.0;
    for (int e = threadIdx.x; e < a.experts; e += kBalanceBlock) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += sums[w][e];
        if (alone) {
            a.prob_sum[e] = s;
            a.counts[e] = count[e];
            l += (double)s * count[e];
        } else {
            a.part_prob[(int64_t)blockIdx.x * a.experts + e] = s;
            a.part_count[(int64_t)blockIdx.x * (a.experts + 1) + e] = count[e];
        }
    }
    if (alone) {
        l = block_sum(l, buf);
        if (threadIdx.x == 0) {
            a.kept[0] = count[a.experts];
            a.loss[0] = loss_of(l, count[a.experts], a.experts, a.k);
        }
    } else if (threadIdx.x == 0) {
        a.part_count[(int64_t)blockIdx.x * (a.experts + 1) + a.experts] = count[a.experts];
        if (blockIdx.x == 0) *a.ticket = 0;
    }
}

// Adds up the blocks' lines: kWide experts a block (the tokens that count are one more column), 1024 / kWide threads each.  Where
// one block has all of them it works the loss out, too; else the block that is done last.
template <int kWide> __global__ __launch_bounds__(1024) void k_balance_sum(BalanceForward a, int32_t lines) {
    constexpr int kDeep = 1024 / kWide;
    __shared__ float prob[kDeep][kWide + 1];
    __shared__ int64_t count[kDeep][kWide + 1];
    __shared__ double buf[16];
    __shared__ bool last;
    const int x = threadIdx.x % kWide, r = threadIdx.x / kWide;
    const int e = blockIdx.x * kWide + x;
    float s = 0.0f;
    int64_t n = 0;
    if (e <= a.experts) {
        const int column = min(e, a.experts - 1);
#pragma unroll 8
        for (int l = r; l < lines; l += kDeep) {
            s += a.part_prob[(int64_t)l * a.experts + column];
            n += a.part_count[(int64_t)l * (a.experts + 1) + e];
        }
    }
    prob[r][x] = s;
    count[r][x] = n;
    for (int d = kDeep / 2; d >= 1; d >>= 1) {
        __syncthreads();
        if (r < d) { prob[r][x] += prob[r + d][x]; count[r][x] += count[r + d][x]; }
    }
    __syncthreads();
    if (r == 0 && e <= a.experts) {
        if (e < a.experts) {
            a.prob_sum[e] = prob[0][x];
            a.counts[e] = count[0][x];
        } else {
            a.kept[0] = count[0][x];
        }
    }
    double l = 0.0;
    if (gridDim.x == 1) {
        if (r == 0 && e < a.experts) l = (double)prob[0][x] * (double)count[0][x];
        l = block_sum(l, buf);
        if (threadIdx.x == 0) a.loss[0] = loss_of(l, count[0][a.experts], a.experts, a.k);
        return;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int q = threadIdx.x; q < a.experts; q += 1024) l += (double)a.prob_sum[q] * (double)a.counts[q];
    l = block_sum(l, buf);
    if (threadIdx.x == 0) a.loss[0] = loss_of(l, a.kept[0], a.experts, a.k);
}

__global__ __launch_bounds__(kBalanceBlock) void k_balance_loss(const int64_t* counts, const float* prob_sum, const int64_t* kept, int32_t experts,
                                                                int32_t k, float* loss) {
    __shared__ double buf[kBalanceBlock / 64];
    double l = 0.0;
    for (int q = threadIdx.x; q < experts; q += kBalanceBlock) l += (double)prob_sum[q] * (double)counts[q];
    l = block_sum(l, buf);
    if (threadIdx.x == 0) loss[0] = loss_of(l, kept[0], experts, k);
}

// Backward.  The gates' gradients of a token go to their experts' places in a row of LDS of the token's lanes, which hold zeros
// otherwise and are cleared again after use; only the token's own lanes, which are of one wavefront, touch that row.
template <typename T, int kLanes, int kItems> __global__ __launch_bounds__(kBalanceBlock, 4) void k_balance_backward(BalanceBackward a) {
    typedef Row<T, kLanes, kItems> R;
    constexpr int kTokens = kBalanceBlock / kLanes;
    __shared__ float extra[kTokens][R::kPitch];
    const int lane = threadIdx.x % kLanes;
    float* slots = extra[threadIdx.x / kLanes];
    const double kept = (double)a.kept[0];
    const double c = kept > 0 ? (a.dloss ? (double)a.dloss[0] : 1.0) * a.experts / (a.k * kept * kept) : 0.0;
    float w[kItems];
    int from[kItems];                                      // this lane's values in the row
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int e = R::place(lane, a.experts, i);
        w[i] = e < a.experts ? (float)(c * (double)a.counts[e]) : 0.0f;
        from[i] = R::slot(e);
        slots[i * kLanes + lane] = 0.0f;
    }
    const int64_t stride = (int64_t)gridDim.x * kTokens, start = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes;
    // A token's logits, and of its choices this lane's first, are asked for while the one before it is worked on.
    R next;
    bool next_keep = false;
    int32_t next_expert = -1;
    float next_dgate = 0.0f;
    auto ask = [&](int64_t t) {
        const int64_t at = t < a.tokens ? t : a.tokens - 1;
        next.load(static_cast<const T*>(a.logits) + at * a.stride, lane, a.experts);
        next_keep = !a.keep || a.keep[at];
        if (a.dgate && lane < a.k) {
            next_expert = a.expert[at * a.k + lane];
            next_dgate = a.dgate[at * a.k + lane];
        }
    };
    if (a.tokens > 0) ask(start);
    for (int64_t t = start; t < a.tokens; t += stride) {
        const bool keep = next_keep;
        const uint32_t expert = (uint32_t)next_expert;
        const float dgate = next_dgate;
        float p[kItems], m = -INFINITY;
        next.get(p);
        ask(t + stride);
        wavefront_exchange();                              // (the row is clear)
        if (expert < (uint32_t)a.experts) atomicAdd(&slots[R::slot(expert)], dgate);
        if (a.dgate)
            for (int i = lane + kLanes; i < a.k; i += kLanes) {
                const uint32_t e = (uint32_t)a.expert[t * a.k + i];
                if (e < (uint32_t)a.experts) atomicAdd(&slots[R::slot(e)], a.dgate[t * a.k + i]);
            }
        bool any = false;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            m = fmaxf(m, p[i]);
            any |= p[i] != -INFINITY;
        }
        m = group_max<kLanes>(m);
        const bool on = keep && group_reduce<kLanes>((uint32_t)any, [](uint32_t x, uint32_t y) { return x | y; }) != 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) p[i] = exp_of(p[i], m);
        const float inv = __builtin_amdgcn_rcpf(group_sum<kLanes>(R::sum_once(lane, a.experts, p)));
        wavefront_exchange();                              // (all gradients are in the row)
        float u[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) u[i] = slots[from[i]];
        float pu[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            u[i] += w[i];
            p[i] *= inv;
            pu[i] = p[i] * u[i];
        }
        const float dot = group_sum<kLanes>(R::sum_once(lane, a.experts, pu));
        wavefront_exchange();                              // (the row has been read)
        if (expert < (uint32_t)a.experts) slots[R::slot(expert)] = 0.0f;
        if (a.dgate)
            for (int i = lane + kLanes; i < a.k; i += kLanes) {
                const uint32_t e = (uint32_t)a.expert[t * a.k + i];
                if (e < (uint32_t)a.experts) slots[R::slot(e)] = 0.0f;
            }
        float o[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) o[i] = on ? p[i] * (u[i] - dot) : 0.0f;
        R::store(static_cast<T*>(a.dlogits) + t * a.dlogits_stride, lane, a.experts, o);
    }
}

// Lanes of a token and a lane's logits: 8, and from 129 experts on 16.  (A call for 131072 16-bit tokens over 256 experts takes 45 us with
// 16 and 57 with 8, for 65536 fp32 tokens over 512 103 with either; 32 do not stay in registers with their keys and sums.)
struct RowShape { int lanes, items; };
RowShape row_shape(int32_t experts) {
    RowShape r = {1, experts <= 128 ? 8 : 16};
    while (r.lanes * r.items < experts) r.lanes *= 2;
    return r;
}
int64_t balance_blocks(int64_t tokens, int32_t experts) {
    return std::max<int64_t>(1, std::min(ceil_div(tokens, kBalanceBlock / row_shape(experts).lanes), kBalanceBlocks));
}

#define P2_BALANCE_CASE(KERNEL, T, LANES, ITEMS) \
    case LANES * 32 + ITEMS: KERNEL<T, LANES, ITEMS><<<grid, dim3(kBalanceBlock), 0, s>>>(a); break;
#define P2_BALANCE_CASES(KERNEL, T)                                                     \
    const RowShape shape = row_shape(a.experts);                                \
    switch (shape.lanes * 32 + shape.items) {                                           \
        P2_BALANCE_CASE(KERNEL, T, 1, 8)                                                \
        P2_BALANCE_CASE(KERNEL, T, 2, 8)                                                \
        P2_BALANCE_CASE(KERNEL, T, 4, 8)                                                \
        P2_BALANCE_CASE(KERNEL, T, 8, 8)                                                \
        P2_BALANCE_CASE(KERNEL, T, 16, 8)                                               \
        P2_BALANCE_CASE(KERNEL, T, 16, 16)                                              \
        P2_BALANCE_CASE(KERNEL, T, 32, 16)                                              \
        P2_BALANCE_CASE(KERNEL, T, 64, 16)                                              \
    }

}  // namespace

int64_t balance_forward_partials(int64_t tokens, int32_t experts) { return balance_blocks(tokens, experts); }

hipError_t launch_balance_forward(const BalanceForward& a, hipStream_t s) {
    const int64_t blocks = balance_blocks(a.tokens, a.experts);
    const dim3 grid((unsigned)blocks);
    if (a.type == P2_F32) { P2_BALANCE_CASES(k_balance_forward, float) }
    else if (a.type == P2_BF16) { P2_BALANCE_CASES(k_balance_forward, bf16_t) }
    else { P2_BALANCE_CASES(k_balance_forward, half_t) }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    if (a.experts < 64) k_balance_sum<64><<<dim3(1), dim3(1024), 0, s>>>(a, (int32_t)blocks);
    else k_balance_sum<16><<<dim3((unsigned)ceil_div(a.experts + 1, 16)), dim3(1024), 0, s>>>(a, (int32_t)blocks);
    return hipGetLastError();
}

hipError_t launch_balance_loss(const int64_t* counts, const float* prob_sum, const int64_t* kept, int32_t experts, int32_t k, float* loss, hipStream_t s) {
    k_balance_loss<<<dim3(1), dim3(kBalanceBlock), 0, s>>>(counts, prob_sum, kept, experts, k, loss);
    return hipGetLastError();
}

hipError_t launch_balance_backward(const BalanceBackward& a, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const dim3 grid((unsigned)balance_blocks(a.tokens, a.experts));
    if (a.type == P2_F32) { P2_BALANCE_CASES(k_balance_backward, float) }
    else if (a.type == P2_BF16) { P2_BALANCE_CASES(k_balance_backward, bf16_t) }
    else { P2_BALANCE_CASES(k_balance_backward, half_t) }
    return hipGetLastError();
}

}  // namespace p2
