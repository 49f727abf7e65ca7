// The router's balance: the k best experts of each token, their probabilities, counts and probability sums per expert,
// the balance loss, and the gradient with respect to the logits.
//
// A token's logits are read once and stay in the registers of kLanes lanes, kItems each (a lane holds whole 16-byte
// vectors); a wavefront takes 64 / kLanes tokens at a time.  Choosing goes by keys in which a larger logit, and of equal ones
// the lower index, is the larger whole number: it is exact and does not depend on how the softmax is rounded.
//
// What bounds it: the gradient, memory (131072 bf16 tokens over 256 experts 29.9 us, 4.8 TB/s; a copy of 4 GiB reaches 4.84).  The choice,
// vector instructions: 395 of them and 16 exponentials for four tokens, 24 of 31.5 us at eight choices of 256 (75 MB: 2.4 TB/s), 6.4 more for the sums
// over blocks (both under the profiler); a call 35.8.  One token: 4.9 us on the device in a call of 9.1.
#include <algorithm>
#include <type_traits>

#include "p2_train_dev.h"

namespace p2 {

namespace {

constexpr int kBalanceBlock = 512;
constexpr int64_t kBalanceBlocks = 512;                // two blocks a compute unit
constexpr float kLog2e = 1.44269504088896340736f;

// Exponentials and inverses of sums are the instructions for 2^x and 1 / x, which are off by a step of 32 bits at most; a library's exponential and a
// division, by half a step each, would take several times their instructions in kernels that vector instructions bound (and half a step of a sum is
// what adding it up rounds off anyway).  Gates are off by 6.8e-8 to 7.2e-8 of their value (root mean square; logits of a spread of 1.5, 8 to 256 experts),
// with these 5.0e-8 to 5.4e-8; probability sums of 20000 tokens by 2.2e-7 at most, with these 3.6e-7 (torch's order of sums).

// e^(v - m), v and m finite or not.
__device__ __forceinline__ float exp_of(float v, float m) { return __builtin_amdgcn_exp2f((v - m) * kLog2e); }

// Keys: whole numbers in the order of the logits, and of equal ones in the order of falling indexes; never 0.  A float's bits, turned
// over where it is negative, are in its order (NaN aside: with_nan puts it above everything).  -0 is 0; what is not above -inf (kNone)
// is never chosen.  16-bit logits and their indexes share 32 bits, 32-bit ones take 64.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
// Two 16-bit logits at a time: sign and magnitude become two's complement, which has one 0, and the sign is turned over.
__device__ __forceinline__ uint32_t ordered_pair(uint32_t w) {
    typedef int16_t short2_t __attribute__((ext_vector_type(2)));
    const short2_t sign = __builtin_bit_cast(short2_t, w) >> 15;
    const uint32_t turned = w ^ (__builtin_bit_cast(uint32_t, sign) | 0x80008000u);
    return __builtin_bit_cast(uint32_t, (short2_t)(__builtin_bit_cast(short2_t, turned) - sign));
}
template <typename T> struct Key {                     // half_t, bf16_t
    typedef uint32_t type;
    static constexpr uint32_t kInf = std::is_same<T, half_t>::value ? 0x7c00u : 0x7f80u;
    static constexpr type kNone = (0x8000u - kInf) << 16;                  // -inf's, without an index
    static __device__ __forceinline__ type with_nan(type k) { return k > ((0x8000u + kInf) << 16 | 0xffffu) || k < kNone ? k | 0xffff0000u : k; }
    static __device__ __forceinline__ bool real(type k) { return k > (kNone | 0xffffu); }
    static __device__ __forceinline__ int index(type k) { return (int)(0xffffu - (k & 0xffffu)); }
    static __device__ __forceinline__ float value(type k) {
        const int v = (int)(k >> 16) - 0x8000;
        return (float)__builtin_bit_cast(T, (uint16_t)(v < 0 ? 0x8000 - v : v));
    }
    // of a vector's N values, the first of which is expert e's (N even)
    template <int N> static __device__ __forceinline__ void of(const vec_t<T, N>& v, int e, type* key) {
        typedef uint32_t words_t __attribute__((ext_vector_type(N / 2)));
        const words_t w = __builtin_bit_cast(words_t, v);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const uint32_t o = ordered_pair(w[j]), low = 0xffffu - (uint32_t)(e + 2 * j);
            key[2 * j] = o << 16 | low;
            key[2 * j + 1] = (o & 0xffff0000u) | (low - 1);
        }
    }
};
template <> struct Key<float> {
    typedef uint64_t type;
    static constexpr uint32_t kBelow = 0x007fffffu;    // ordered(-inf)
    static constexpr type kNone = (uint64_t)kBelow << 32;
    static __device__ __forceinline__ type with_nan(type k) {
        const uint32_t o = (uint32_t)(k >> 32);
        return o > 0xff800000u || o < kBelow ? k | 0xffffffff00000000ull : k;
    }
    static __device__ __forceinline__ bool real(type k) { return (uint32_t)(k >> 32) > kBelow; }
    static __device__ __forceinline__ int index(type k) { return (int)(0xffffffffu - (uint32_t)k); }
    static __device__ __forceinline__ float value(type k) {
        const uint32_t o = (uint32_t)(k >> 32);
        return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
    }
    template <int N> static __device__ __forceinline__ void of(const vec_t<float, N>& v, int e, type* key) {
#pragma unroll
        for (int j = 0; j < N; ++j) key[j] = (uint64_t)ordered(v[j]) << 32 | (0xffffffffu - (uint32_t)(e + j));
    }
};

// A lane's kAhead largest keys in falling order; 0 where it has fewer.  insert(key, i): the lane's i-th, in the order of their experts,
// among the first kDepth.
template <typename K, int kAhead = 4> struct Largest { // 32 bits: the middle of three in an instruction each
    static constexpr int kMost = kAhead;
    K v[kAhead] = {};
    template <int kDepth> __device__ __forceinline__ void insert(K x, int) {
#pragma unroll
        for (int n = kDepth - 1; n > 0; --n) v[n] = max(min(v[n - 1], v[n]), min(max(v[n - 1], v[n]), x));
        v[0] = max(v[0], x);
    }
    __device__ __forceinline__ bool empty() const { return v[0] == 0; }
    template <typename R> __device__ __forceinline__ K first(int, int) const { return v[0]; }
    __device__ __forceinline__ void pop() {
#pragma unroll
        for (int n = 0; n + 1 < kAhead; ++n) v[n] = v[n + 1];
        v[kAhead - 1] = 0;
    }
};
template <> struct Largest<uint64_t> {                 // values, and which of the lane's they are: of equal ones the first
    static constexpr int kAhead = 3, kMost = kAhead;       // (four: 4 % more time for 8 of 512 experts, registers spill)
    Largest<uint32_t, kAhead> value;
    uint32_t of[kAhead] = {};
    template <int kDepth> __device__ __forceinline__ void insert(uint64_t x, int i) {
        const uint32_t o = (uint32_t)(x >> 32);
#pragma unroll
        for (int n = kDepth - 1; n >= 0; --n) of[n] = n > 0 && o > value.v[n > 0 ? n - 1 : 0] ? of[n > 0 ? n - 1 : 0] : o > value.v[n] ? i : of[n];
        value.template insert<kDepth>(o, i);
    }
    __device__ __forceinline__ bool empty() const { return value.empty(); }
    template <typename R> __device__ __forceinline__ uint64_t first(int lane, int experts) const {
        return (uint64_t)value.v[0] << 32 | (0xffffffffu - (uint32_t)R::place(lane, experts, (int)of[0]));
    }
    __device__ __forceinline__ void pop() {
        value.pop();
#pragma unroll
        for (int n = 0; n + 1 < kAhead; ++n) of[n] = of[n + 1];
        of[kAhead - 1] = 0;
    }
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
    __device__ __forceinline__ void keys(int lane, int experts, typename Key<T>::type (&key)[kItems]) const {
#pragma unroll
        for (int q = 0; q < kVecs; ++q) Key<T>::template of<V>(raw[q], place(lane, experts, q * V), &key[q * V]);
        count_once(lane, experts, Key<T>::kNone, key);
    }
    // `other` in the place of values that are not this lane's to count
    template <typename U> static __device__ __forceinline__ void count_once(int lane, int experts, U other, U (&p)[kItems]) {
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

// p = softmax of a token's logits; expert, gate: its k largest; per block counts of choices and sums of p.
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
    auto logits_of = [&](int64_t t) { return static_cast<const T*>(a.logits) + (t < a.tokens ? t : a.tokens - 1) * a.stride; };
    auto ask = [&](int64_t t) {
        next.load(logits_of(t), lane, a.experts);
        next_keep = t < a.tokens && (!a.keep || a.keep[t]);
    };
    const int64_t first = (int64_t)blockIdx.x * kTokens;
    if (first < a.tokens) ask(first + threadIdx.x / kLanes);
    for (int64_t t0 = first; t0 < a.tokens; t0 += stride) {
        const int64_t t = t0 + threadIdx.x / kLanes;
        const bool there = t < a.tokens, keep = next_keep;
        float p[kItems];
        next.get(p);
        auto larger = [](K x, K y) { return x > y ? x : y; };
        Largest<K> mine;
        {
            K key[kItems];
            next.keys(lane, a.experts, key);
            if (a.k <= 2) {                                // (131072 tokens, 2 of 256 experts: 27.4 us for 28.6)
#pragma unroll
                for (int i = 0; i < kItems; ++i) mine.template insert<2>(key[i], i);
            } else {
#pragma unroll
                for (int i = 0; i < kItems; ++i) mine.template insert<Largest<K>::kMost>(key[i], i);
            }
        }
        if (t0 + stride < a.tokens) ask(t + stride);
        auto best_of_all = [&] { return group_reduce<kLanes>(mine.template first<R>(lane, a.experts), larger); };
        K best = best_of_all();
        // e^(v - m) as 2^(v log2e - m log2e): what the rounding of the second product is off by is common to the row.
        float m = Key<T>::value(best);
        const float shift = m * kLog2e;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], kLog2e, -shift));
        R::count_once(lane, a.experts, 0.0f, p);
#pragma unroll
        for (int i = 0; i < kItems; ++i) s += p[i];
        s = group_sum<kLanes>(s);
        // Logits whose products overflow or are off by more than a factor, infinities and NaN: from the differences, NaN above everything.
        const bool odd = !(s > 0.5f && s < 2.0f * P2_MAX_EXPERTS);
        if (odd) {
            mine = Largest<K>();
            K key[kItems];
            R again;
            again.load(logits_of(t), lane, a.experts);
            again.keys(lane, a.experts, key);
            again.get(p);
#pragma unroll
            for (int i = 0; i < kItems; ++i) mine.template insert<Largest<K>::kMost>(Key<T>::with_nan(key[i]), i);
            best = best_of_all();
            m = Key<T>::value(best);
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < kItems; ++i) p[i] = exp_of(p[i], m);
            R::count_once(lane, a.experts, 0.0f, p);       // (m may be -inf)
#pragma unroll
            for (int i = 0; i < kItems; ++i) s += p[i];
            s = group_sum<kLanes>(s);
        }
        const float inv = __builtin_amdgcn_rcpf(s);
        const bool on = keep && Key<T>::real(best);
        if (on) {
            if (lane == 0) atomicAdd(&count[a.experts], 1);
#pragma unroll
            for (int i = 0; i < kItems; ++i) acc[i] += p[i] * inv;
        }
        // The k best, one after the other: the largest of what the lanes have left.  A lane that has given all of its list looks for
        // the next ones among its keys below the last (of 256 experts' eight best 1 token in 60 has four in one lane, 1 in 5 three).  Lane i keeps the i-th of as
        // many as there are lanes, which are then written.
        auto advance = [&] {
            if (mine.template first<R>(lane, a.experts) == best) mine.pop();
            if (__any(mine.empty())) {
                K key[kItems];
                R again;
                again.load(logits_of(t), lane, a.experts);
                again.keys(lane, a.experts, key);
                if (mine.empty())
#pragma unroll
                    for (int q = 0; q < kItems; ++q) {
                        const K x = odd ? Key<T>::with_nan(key[q]) : key[q];
                        mine.template insert<Largest<K>::kMost>(x < best ? x : 0, q);
                    }
            }
            best = best_of_all();
        };
        for (int base = 0; base < a.k; base += kLanes) {
            const int n = min(a.k - base, kLanes);
            if (base) advance();
            K held = best;
            for (int i = 1; i < n; ++i) {
                advance();
                if (lane >= i) held = best;
            }
            if (there && lane < n) {
                const bool real = keep && Key<T>::real(held);
                const int e = Key<T>::index(held);
                const float v = Key<T>::value(held);
                const int64_t at = t * a.k + base + lane;
                a.expert[at] = real ? e : -1;
                a.gate[at] = real ? (odd ? exp_of(v, m) : __builtin_amdgcn_exp2f(fmaf(v, kLog2e, -shift))) * inv : 0.0f;
                if (real) atomicAdd(&count[e], 1);
            }
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
    __shared__ float prob[16][kWide];
    __shared__ int64_t count[16][kWide], tokens;
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
    // a wavefront's lanes of the same expert, then the wavefronts
#pragma unroll
    for (int d = kWide; d < 64; d <<= 1) { s += __shfl_xor(s, d, 64); n += __shfl_xor(n, d, 64); }
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) < kWide) { prob[wave][x] = s; count[wave][x] = n; }
    __syncthreads();
    if (r == 0) {
        s = 0.0f;
        n = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) { s += prob[w][x]; n += count[w][x]; }
        if (e < a.experts) {
            a.prob_sum[e] = s;
            a.counts[e] = n;
        } else if (e == a.experts) {
            a.kept[0] = n;
            tokens = n;
        }
    }
    double l = 0.0;
    if (gridDim.x == 1) {
        if (r == 0 && e < a.experts) l = (double)s * (double)n;
        l = block_sum(l, buf);
        if (threadIdx.x == 0) a.loss[0] = loss_of(l, tokens, a.experts, a.k);
        return;
    }
    __syncthreads();
    // (thread 0's wavefront has written all of the block's results)
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
    __syncthreads();
    if (!last) return;
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

// Backward.  u = dloss experts / (k kept^2) counts + the choices' dgate, dlogits = p (u - sum p u).  The gates' gradients of a token go to their experts' places in a row of LDS of the token's lanes, which hold zeros
// otherwise and are cleared again after use; only the token's own lanes, which are of one wavefront, touch that row.  Where a caller's choices name
// an expert more than once (the forward pass never does) its gradients are added one by one in the order of the choices: instructions of one wavefront
// follow each other, and an instruction's additions to one place are made in the order of the lanes, which a test of sums that cancel only in that
// order holds to.
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

// Lanes of a token and a lane's logits: 8, and from 129 experts on 16, in both passes (us of the forward pass / of the gradient, with 8 against 16 logits
// a lane): 131072 tokens over 64 experts, bf16 and two choices 16 / 11 against 16 / 14, eight 21 / 12 against 27 / 17, fp32 35 / 14 against 50 / 18;
// over 128, eight choices, bf16 28 / 18 against 28 / 19, fp32 48 / 26 against 64 / 28; over 160 bf16 50 / 32 against 38 / 29; over 256 bf16 49 / 32
// against 37 / 29, fp32 81 / 46 against 81 / 46 (two choices 46 / 46 against 56 / 45: the one kind that 8 would suit better); 65536 over 512 bf16
// 53 / 33 against 38 / 30, fp32 88 / 46 against 75 / 46.
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
