// What the training operators' kernels share: element types, loads of whole vectors from rows of any alignment,
// reductions over groups of lanes, and the launch entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "../../include/p2_train.h"

namespace p2 {

int32_t api_fail(int32_t code, const std::string& text);      // p2_api.hip: the calling thread's last error
int32_t api_hip_fail(hipError_t e, const char* what);

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t type_bytes(int32_t type) { return type == P2_F32 ? 4 : 2; }

typedef _Float16 half_t;
typedef __bf16 bf16_t;

// N elements from an address that is aligned to one of them: the device reads unaligned 16-byte words in one
// instruction, so rows of odd lengths and strides need no variant of their own.
template <typename T, int N> struct Vec {
    typedef T type __attribute__((ext_vector_type(N), aligned(alignof(T))));
};
template <typename T, int N> using vec_t = typename Vec<T, N>::type;

template <typename T, int N> __device__ __forceinline__ void load_vec(const T* p, float (&v)[N]) {
    const vec_t<T, N> r = *reinterpret_cast<const vec_t<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)r[i];
}
template <typename T, int N> __device__ __forceinline__ void store_vec(T* p, const float (&v)[N]) {
    vec_t<T, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = (T)v[i];
    *reinterpret_cast<vec_t<T, N>*>(p) = r;
}
// The first `n` of N elements (n may be <= 0 or >= N); the others are `other`.
template <typename T, int N> __device__ __forceinline__ void load_part(const T* p, int64_t n, float (&v)[N], float other) {
    if (n >= N) { load_vec<T, N>(p, v); return; }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? (float)p[i] : other;
}
template <typename T, int N> __device__ __forceinline__ void store_part(T* p, int64_t n, const float (&v)[N]) {
    if (n >= N) { store_vec<T, N>(p, v); return; }
#pragma unroll
    for (int i = 0; i < N; ++i) if (i < n) p[i] = (T)v[i];
}

// A lane's N elements of a row, from column c on (N <= cols).  The load is always a whole vector inside the row and depends on
// nothing, so that many of them are under way together.  Where the row's end cuts the vector, or lies before it, the last N elements are
// taken instead: those before column c are another lane's, too.  They count once, for that lane; what a lane makes of them is
// the same, so whole vectors are stored as well.
__device__ __forceinline__ int vec_at(int c, int cols, int n) { return min(c, cols - n); }
template <typename T, int N> __device__ __forceinline__ vec_t<T, N> load_whole(const T* row, int c, int cols) {
    return *reinterpret_cast<const vec_t<T, N>*>(row + vec_at(c, cols, N));
}
// Whether element j of the vector is this lane's.  kWhole: the row is whole vectors, and the lane has all of its own or none.
template <int N, bool kWhole> __device__ __forceinline__ bool own(int c, int cols, int j) {
    return kWhole ? c < cols : j >= c - vec_at(c, cols, N);
}

// Weights have a type of their own, which the whole launch agrees on.
template <int N> __device__ __forceinline__ void load_typed(const void* p, int32_t type, int64_t at, int64_t n, float (&v)[N], float other) {
    if (type == P2_F32) load_part<float, N>(static_cast<const float*>(p) + at, n, v, other);
    else if (type == P2_BF16) load_part<bf16_t, N>(static_cast<const bf16_t*>(p) + at, n, v, other);
    else load_part<half_t, N>(static_cast<const half_t*>(p) + at, n, v, other);
}
__device__ __forceinline__ void store_typed(void* p, int32_t type, int64_t at, float v) {
    if (type == P2_F32) static_cast<float*>(p)[at] = v;
    else if (type == P2_BF16) static_cast<bf16_t*>(p)[at] = (bf16_t)v;
    else static_cast<half_t*>(p)[at] = (half_t)v;
}

// A value of another lane of the same 16, without a detour through LDS: kStep 1 and 2 exchange lanes 1 and 2 apart, 4 and 8 mirror
// groups of 8 and 16 lanes, which for a reduction over lanes that already agree in groups of 4 and 8 is as good.
template <int kStep> __device__ __forceinline__ uint32_t neighbour(uint32_t v) {
    constexpr int kControl = kStep == 1 ? 0xb1 : kStep == 2 ? 0x4e : kStep == 4 ? 0x141 : 0x140;
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kControl, 0xf, 0xf, true);
}
template <int kStep> __device__ __forceinline__ float neighbour(float v) { return __uint_as_float(neighbour<kStep>(__float_as_uint(v))); }
template <int kStep> __device__ __forceinline__ uint64_t neighbour(uint64_t v) {
    return (uint64_t)neighbour<kStep>((uint32_t)(v >> 32)) << 32 | neighbour<kStep>((uint32_t)v);
}
// A reduction's step over lanes 16 (32) apart: the instruction exchanges every second row of 16 lanes (half of 32) of two registers, so
// that of a value and itself one register has the lower lanes' values twice, the other the upper lanes'.
template <int kFar, typename F> __device__ __forceinline__ uint32_t far_step(uint32_t v, F&& f) {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (kFar == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return f((uint32_t)r[0], (uint32_t)r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return f((uint32_t)r[0], (uint32_t)r[1]);
    }
#else
    return f(v, v);
#endif
}
template <int kFar, typename F> __device__ __forceinline__ float far_step(float v, F&& f) {
    return __uint_as_float(far_step<kFar>(__float_as_uint(v), [&](uint32_t a, uint32_t b) { return __float_as_uint(f(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int kFar, typename F> __device__ __forceinline__ uint64_t far_step(uint64_t v, F&& f) {
    uint32_t other_low = 0, low = 0;
    far_step<kFar>((uint32_t)v, [&](uint32_t a, uint32_t b) { low = a; other_low = b; return a; });
    uint32_t other_high = 0, high = 0;
    far_step<kFar>((uint32_t)(v >> 32), [&](uint32_t a, uint32_t b) { high = a; other_high = b; return a; });
    return f((uint64_t)high << 32 | low, (uint64_t)other_high << 32 | other_low);
}

// Reduction over groups of L consecutive lanes (a power of two up to 64); every lane gets the result, always in one order.
template <int L, typename V, typename F> __device__ __forceinline__ V group_reduce(V v, F&& f) {
    if constexpr (L >= 2) v = f(v, neighbour<1>(v));
    if constexpr (L >= 4) v = f(v, neighbour<2>(v));
    if constexpr (L >= 8) v = f(v, neighbour<4>(v));
    if constexpr (L >= 16) v = f(v, neighbour<8>(v));
    if constexpr (L >= 32) v = far_step<16>(v, f);
    if constexpr (L >= 64) v = far_step<32>(v, f);
    return v;
}
template <int L> __device__ __forceinline__ float group_sum(float v) {
    return group_reduce<L>(v, [](float a, float b) { return a + b; });
}
template <int L> __device__ __forceinline__ float group_max(float v) {
    return group_reduce<L>(v, [](float a, float b) { return fmaxf(a, b); });
}

// What the wavefront's lanes have written to LDS is there for its other lanes.
__device__ __forceinline__ void wavefront_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct NormForward {
    const void* x; const void* weight; const void* bias; void* y; float* mean; float* rstd;
    int64_t x_stride, y_stride, rows, cols;
    float eps;
    int32_t type, weight_type;
};
hipError_t launch_norm_forward(const NormForward& a, hipStream_t stream);

struct NormBackward {
    const void* dy; const void* x; const void* weight; const float* mean; const float* rstd; void* dx; void* dweight; void* dbias;
    float* partial;                   // [blocks][2][cols]; NULL: neither dweight nor dbias
    int64_t dy_stride, x_stride, dx_stride, rows, cols;
    int32_t type, weight_type;
};
int64_t norm_backward_partials(int64_t rows, int64_t cols);
hipError_t launch_norm_backward(const NormBackward& a, hipStream_t stream);

struct BalanceForward {
    const void* logits; const uint8_t* keep; int32_t* expert; float* gate; int64_t* counts; float* prob_sum; int64_t* kept; float* loss;
    float* part_prob;                 // [blocks][experts]
    int32_t* part_count;              // [blocks][experts + 1], the last one: tokens that count
    uint32_t* ticket;                 // blocks of the summing kernel that are done
    int64_t stride, tokens;
    int32_t experts, k, type;
};
int64_t balance_forward_partials(int64_t tokens, int32_t experts);
hipError_t launch_balance_forward(const BalanceForward& a, hipStream_t stream);
hipError_t launch_balance_loss(const int64_t* counts, const float* prob_sum, const int64_t* kept, int32_t experts, int32_t k, float* loss, hipStream_t stream);

struct BalanceBackward {
    const void* logits; const uint8_t* keep; const int32_t* expert; const float* dgate; const int64_t* counts; const int64_t* kept;
    const float* dloss; void* dlogits;
    int64_t stride, dlogits_stride, tokens;
    int32_t experts, k, type;
};
hipError_t launch_balance_backward(const BalanceBackward& a, hipStream_t stream);

struct Orthogonalize {
    const void* g; void* out; void* workspace;
    int64_t stride, matrix_stride, count, rows, cols, out_stride, out_matrix_stride;
    int32_t type, out_type, steps;
    double a, b, c, eps, scale;
    const double* bounds;             // [steps + 1]: what the singular values stay below before each step
};
// Fills bounds[0 .. steps]; false where the iterates may grow past what the call takes.
bool orthogonalize_bounds(const Orthogonalize& a, double* bounds);
int64_t orthogonalize_workspace(int64_t count, int64_t rows, int64_t cols);
hipError_t launch_orthogonalize(const Orthogonalize& a, hipStream_t stream);

}  // namespace p2
