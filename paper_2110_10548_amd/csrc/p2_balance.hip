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
// over where it is negative, are in its order.  16-bit logits leave the lowest 13 of them unused: the index goes there; for 32-bit
// ones it takes 32 bits more.  -0 is 0, NaN above everything; what is not above -inf (kNone) is never chosen.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t b = __float_as_uint(f + 0.0f);
    const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return f != f ? 0xffffffffu : o;
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
constexpr uint32_t kNone = 0x007fffffu;                // ordered(-inf)
template <typename T> struct Key {                     // half_t, bf16_t
    typedef uint32_t type;
    static constexpr uint32_t kLow = 0x1fffu;
    static __device__ __forceinline__ type of(float f, int e) { return (ordered(f) & ~kLow) | (kLow - (uint32_t)e); }
    static __device__ __forceinline__ bool real(type k) { return (k & ~kLow) > (kNone & ~kLow); }
    static __device__ __forceinline__ int index(type k) { return (int)(kLow - (k & kLow)); }
    static __device__ __forceinline__ float value(type k) { return from_ordered(k & 0x80000000u ? k & ~kLow : k | kLow); }
};
template <> struct Key<float> {
    typedef uint64_t type;
    static __device__ __forceinline__ type of(float f, int e) { return (uint64_t)ordered(f) << 32 | (0xffffffffu - (uint32_t)e); }
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

// The logits of a row as this lane's kItems, -inf where there are none.
template <typename T, int kLanes, int kItems> struct Row {
    static constexpr int V = 16 / sizeof(T) < kItems ? 16 / sizeof(T) : kItems;
    static constexpr int kVecs = kItems / V;
    static __device__ __forceinline__ int at(int lane, int i) { return ((i / V) * kLanes + lane) * V + i % V; }
    static __device__ __forceinline__ void load(const T* row, int lane, int experts, T (&z)[kItems]) {
#pragma unroll
        for (int q = 0; q < kVecs; ++q) {
            const int e = (q * kLanes + lane) * V;
            if (e + V <= experts) {
                const vec_t<T, V> r = *reinterpret_cast<const vec_t<T, V>*>(row + e);
#pragma unroll
                for (int j = 0; j < V; ++j) z[q * V + j] = r[j];
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) z[q * V + j] = e + j < experts ? row[e + j] : (T)-INFINITY;
            }
        }
    }
};

template <typename T, int kLanes, int kItems> __global__ __launch_bounds__(kBalanceBlock) void k_balance_forward(BalanceForward a) {
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
    for (int64_t t0 = (int64_t)blockIdx.x * kTokens; t0 < a.tokens; t0 += (int64_t)gridDim.x * kTokens) {
        const int64_t t = t0 + threadIdx.x / kLanes;
        const bool there = t < a.tokens;
        const bool keep = there && (!a.keep || a.keep[t]);
        float p[kItems];
        K key[kItems];
        {
            T z[kItems];
            R::load(static_cast<const T*>(a.logits) + (there ? t : a.tokens - 1) * a.stride, lane, a.experts, z);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                p[i] = (float)z[i];
                key[i] = Key<T>::of(p[i], R::at(lane, i));
            }
        }
        float m = p[0];
#pragma unroll
        for (int i = 1; i < kItems; ++i) m = fmaxf(m, p[i]);
        m = group_max<kLanes>(m);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            p[i] = R::at(lane, i) < a.experts ? exp_of(p[i], m) : 0.0f;
            s += p[i];
        }
        const float inv = 1.0f / group_sum<kLanes>(s);
        // The k best, one after the other: the next is the largest key below the last, and as whole numbers that wrap around
        // key - last is the larger the nearer the key is below.  Lane i % kLanes keeps the i-th until as many as there are lanes
        // are to be written.
        int32_t held_expert = -1;
        float held_gate = 0.0f;
        bool on = false;
        K last = 0;
        for (int i = 0; i < a.k; ++i) {
            K best = key[0] - last;
#pragma unroll
            for (int q = 1; q < kItems; ++q) { const K d = key[q] - last; best = d > best ? d : best; }
            best = group_reduce<kLanes>(best, [](K x, K y) { return x > y ? x : y; });
            last += best;                                  // (there are k keys at least: -inf has one, too)
            const bool real = keep && Key<T>::real(last);
            if (i == 0) on = real;
            if (i % kLanes == lane) {
                held_expert = real ? Key<T>::index(last) : -1;
                held_gate = real ? exp_of(Key<T>::value(last), m) * inv : 0.0f;
            }
            if ((i + 1) % kLanes == 0 || i + 1 == a.k) {
                const int slot = i - i % kLanes + lane;
                if (there && slot <= i) {
                    a.expert[t * a.k + slot] = held_expert;
                    a.gate[t * a.k + slot] = held_gate;
                    if (held_expert >= 0) atomicAdd(&count[held_expert], 1);
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
        if ((threadIdx.x & 63) < kLanes) sums[threadIdx.x >> 6][R::at(lane, i)] = acc[i];
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

// Adds up the blocks' lines: 16 experts a block (the tokens that count are one more column), 64 threads each.  The block
// that is done last works the loss out.
__global__ __launch_bounds__(1024) void k_balance_sum(BalanceForward a, int32_t lines) {
    __shared__ float prob[64][17];
    __shared__ int64_t count[64][17];
    __shared__ double buf[16];
    __shared__ bool last;
    const int x = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int e = blockIdx.x * 16 + x;
    float s = 0.0f;
    int64_t n = 0;
    if (e <= a.experts) {
        const int column = min(e, a.experts - 1);
#pragma unroll 8
        for (int l = r; l < lines; l += 64) {
            s += a.part_prob[(int64_t)l * a.experts + column];
            n += a.part_count[(int64_t)l * (a.experts + 1) + e];
        }
    }
    prob[r][x] = s;
    count[r][x] = n;
    for (int d = 32; d >= 1; d >>= 1) {
        __syncthreads();
        if (r < d) { prob[r][x] += prob[r + d][x]; count[r][x] += count[r + d][x]; }
    }
    if (r == 0 && e <= a.experts) {
        if (e < a.experts) {
            a.prob_sum[e] = prob[0][x];
            a.counts[e] = count[0][x];
        } else {
            a.kept[0] = count[0][x];
        }
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
    double l = 0.0;
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
template <typename T, int kLanes, int kItems> __global__ __launch_bounds__(kBalanceBlock) void k_balance_backward(BalanceBackward a) {
    typedef Row<T, kLanes, kItems> R;
    constexpr int kTokens = kBalanceBlock / kLanes;
    constexpr int kWidth = kLanes * kItems;
    __shared__ __attribute__((aligned(16))) float extra[kTokens][kWidth];
    const int lane = threadIdx.x % kLanes;
    float* mine = extra[threadIdx.x / kLanes];
    const double kept = (double)a.kept[0];
    const double c = kept > 0 ? (a.dloss ? (double)a.dloss[0] : 1.0) * a.experts / (a.k * kept * kept) : 0.0;
    float w[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int e = R::at(lane, i);
        w[i] = e < a.experts ? (float)(c * (double)a.counts[e]) : 0.0f;
        mine[e] = 0.0f;
    }
    for (int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes; t < a.tokens; t += (int64_t)gridDim.x * kTokens) {
        T z[kItems];
        R::load(static_cast<const T*>(a.logits) + t * a.stride, lane, a.experts, z);
        const bool keep = !a.keep || a.keep[t];
        wavefront_exchange();                              // (the row is clear)
        if (a.dgate)
            for (int i = lane; i < a.k; i += kLanes) {
                const uint32_t e = (uint32_t)a.expert[t * a.k + i];
                if (e < (uint32_t)a.experts) atomicAdd(&mine[e], a.dgate[t * a.k + i]);
            }
        float p[kItems], m = -INFINITY, any = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            p[i] = (float)z[i];
            m = fmaxf(m, p[i]);
            any = p[i] != -INFINITY ? 1.0f : any;
        }
        m = group_max<kLanes>(m);
        const bool on = keep && group_max<kLanes>(any) > 0.0f;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            p[i] = R::at(lane, i) < a.experts ? exp_of(p[i], m) : 0.0f;
            s += p[i];
        }
        const float inv = 1.0f / group_sum<kLanes>(s);
        wavefront_exchange();                              // (all gradients are in the row)
        float u[kItems], dot = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            u[i] = w[i] + mine[R::at(lane, i)];
            p[i] *= inv;
            dot += p[i] * u[i];
        }
        dot = group_sum<kLanes>(dot);
        wavefront_exchange();                              // (the row has been read)
        if (a.dgate)
            for (int i = lane; i < a.k; i += kLanes) {
                const uint32_t e = (uint32_t)a.expert[t * a.k + i];
                if (e < (uint32_t)a.experts) mine[e] = 0.0f;
            }
        T* out = static_cast<T*>(a.dlogits) + t * a.dlogits_stride;
#pragma unroll
        for (int q = 0; q < R::kVecs; ++q) {
            const int e = (q * kLanes + lane) * R::V;
            float o[R::V];
#pragma unroll
            for (int j = 0; j < R::V; ++j) o[j] = on ? p[q * R::V + j] * (u[q * R::V + j] - dot) : 0.0f;
            store_part<T, R::V>(out + e, a.experts - e, o);
        }
    }
}

// Lanes of a token: 16 at most up to 512 experts (reductions over 16 lanes need no LDS), and a lane's logits 8 to 32.
int lanes_for(int32_t experts) {
    int lanes = 1;
    while (lanes < 16 && lanes * 8 < experts) lanes *= 2;
    return experts <= 512 ? lanes : 64;
}
int64_t balance_blocks(int64_t tokens, int32_t experts) {
    return std::max<int64_t>(1, std::min(ceil_div(tokens, kBalanceBlock / lanes_for(experts)), kBalanceBlocks));
}

#define P2_BALANCE_CASES(KERNEL, T)                                                                       \
    switch (lanes_for(a.experts)) {                                                                       \
        case 1: KERNEL<T, 1, 8><<<grid, dim3(kBalanceBlock), 0, s>>>(a); break;                           \
        case 2: KERNEL<T, 2, 8><<<grid, dim3(kBalanceBlock), 0, s>>>(a); break;                           \
        case 4: KERNEL<T, 4, 8><<<grid, dim3(kBalanceBlock), 0, s>>>(a); break;                           \
        case 8: KERNEL<T, 8, 8><<<grid, dim3(kBalanceBlock), 0, s>>>(a); break;                           \
        case 16:                                                                                          \
            if (a.experts <= 128) KERNEL<T, 16, 8><<<grid, dim3(kBalanceBlock), 0, s>>>(a);               \
            else if (a.experts <= 256) KERNEL<T, 16, 16><<<grid, dim3(kBalanceBlock), 0, s>>>(a);         \
            else KERNEL<T, 16, 32><<<grid, dim3(kBalanceBlock), 0, s>>>(a);                               \
            break;                                                                                        \
        default: KERNEL<T, 64, 16><<<grid, dim3(kBalanceBlock), 0, s>>>(a);                               \
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
    k_balance_sum<<<dim3((unsigned)ceil_div(a.experts + 1, 16)), dim3(1024), 0, s>>>(a, (int32_t)blocks);
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
